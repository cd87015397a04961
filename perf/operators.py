"""Microscaled 4-bit linear layers, the same by expert, and gated activations
with 8-bit checkpoints, as cases to be timed.

``linear``         Y = X W^T.  X comes as the layer's input, W as the microscaled
                   4-bit matrix that a serving program keeps.
``linear_train``   a whole training step of the layer: W and X quantized, Y; then dY
                   quantized along both axes, dX = dY W and dW = dY^T X.
``experts``        ``linear`` with a weight matrix for each of E experts: the rows of X
                   come sorted by expert, expert e's are [offsets[e], offsets[e + 1]).
``experts_train``  ``linear_train`` in the same way; the blocks of dW's inner axis, the
                   rows, start anew at each expert.
``act``            h = act(g) u (or act(x)) and its backward pass from a copy of the
                   input in 8 bits.

Microscaled 4-bit (E2M1 with one power-of-two scale, E8M0, for 32 consecutive
elements of a product's inner axis): scale 2^(s - 127) with s the smallest that
leaves no element of the block more than half a step off, so max |x| / scale <= 7;
element = x / scale rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to
the even code).  The 8-bit copy holds x = code 2^(s - 127), code in [-127, 127],
by the same rule: max |code| < 127.5 before rounding.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

MOST_FLOPS = 6 * 8192 * 4096 * 11008.0      # of the largest listed case
MOST_BYTES = 1.9e9


def listed():
    return [
        # one token through a projection of a 4096-wide model: the weights are all there is to read
        {"name": "linear_token", "kind": "linear", "dtype": "bf16", "M": 1, "K": 4096, "N": 4096},
        # a 1000-way classifier on 2048 features in fp32, a small batch: sizes that no tile divides
        {"name": "linear_classifier", "kind": "linear", "dtype": "f32", "M": 37, "K": 2048, "N": 1000},
        # a prompt of 8192 tokens through the wide projection of an MLP
        {"name": "linear_prefill", "kind": "linear", "dtype": "bf16", "M": 8192, "K": 4096, "N": 11008},
        # an attention projection over 16 sequences of 197 tokens, fp32: an odd row count
        {"name": "linear_train_197", "kind": "linear_train", "dtype": "f32", "M": 16 * 197, "K": 768, "N": 768},
        # the training step of the large linear layer, the benchmark's sizes
        {"name": "linear_train_large", "kind": "linear_train", "dtype": "bf16", "M": 8192, "K": 4096, "N": 11008},
        # one token sent to 8 of 64 experts
        {"name": "experts_token", "kind": "experts", "dtype": "bf16", "M": 8, "K": 2048, "N": 1024, "E": 64, "skew": 0.3},
        # a prompt of 2048 tokens sent to 8 of 64 experts each, uneven loads
        {"name": "experts_prefill", "kind": "experts", "dtype": "bf16", "M": 16384, "K": 2048, "N": 1408, "E": 64,
         "skew": 0.5},
        # a small training batch in fp32, most of it on few experts: widths that no block of 32 divides, empty experts
        {"name": "experts_train_uneven", "kind": "experts_train", "dtype": "f32", "M": 1187, "K": 1000, "N": 520, "E": 12,
         "skew": 1.5},
        # a training step of 16 experts on 32768 routed rows
        {"name": "experts_train_large", "kind": "experts_train", "dtype": "bf16", "M": 32768, "K": 2048, "N": 4096,
         "E": 16, "skew": 0.3},
        # GELU between two layers, 197 tokens, an odd width in fp32
        {"name": "act_gelu_197", "kind": "act", "dtype": "f32", "M": 197, "F": 1000, "act": "gelu", "gated": False},
        # a gated GELU on 2048 tokens
        {"name": "act_geglu", "kind": "act", "dtype": "bf16", "M": 2048, "F": 2752, "act": "gelu", "gated": True},
        # the gated SiLU of the large MLP
        {"name": "act_swiglu_large", "kind": "act", "dtype": "bf16", "M": 8192, "F": 11008, "act": "silu", "gated": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        c = {"kind": rng.choice(["linear", "linear_train", "experts", "experts_train", "act"]),
             "dtype": rng.choice(["bf16", "bf16", "f32"])}
        if c["kind"] == "act":
            c |= {"M": _log_int(rng, 1, 16384), "F": _log_int(rng, 32, 16384), "act": rng.choice(["silu", "gelu"]),
                  "gated": rng.random() < 0.7}
        else:
            c |= {"M": _log_int(rng, 1, 32768), "K": _log_int(rng, 64, 8192), "N": _log_int(rng, 32, 11008)}
            if rng.random() < 0.5:      # widths that are not odd by design: multiples of 64
                c["K"], c["N"] = -(-c["K"] // 64) * 64, -(-c["N"] // 64) * 64
            if c["kind"].startswith("experts"):
                c |= {"E": _log_int(rng, 2, 128), "skew": round(rng.uniform(0.0, 1.5), 2)}
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and _room(c) <= 6e9:
            return c


def _room(c):
    """Bytes of the largest things that a plain form holds."""
    if c["kind"] == "act":
        return 4.0 * c["M"] * c["F"] * 4
    e = c.get("E", 1)
    rows = c["M"] * (1 if e == 1 else min(e, 3 * math.exp(c["skew"])))
    return 4.0 * (rows * (c["K"] + c["N"]) + e * c["K"] * c["N"])


def work(case):
    s = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "act":
        m, f, w = case["M"], case["F"], case["F"] * (2 if case["gated"] else 1)
        # input, h, the 8-bit copy out and in, dh, the gradient
        return {"bytes": m * (w * s + f * s + 2 * w * 33 / 32 + f * s + w * s), "flops": 30.0 * m * f}
    m, k, n = case["M"], case["K"], case["N"]
    e = min(case.get("E", 1), m)        # experts that can have a row
    if case["kind"] in ("linear", "experts"):
        return {"bytes": m * k * s + e * n * k * 17 / 32 + m * n * s, "flops": 2.0 * m * n * k}
    # x, dy, W once; y, dx in their type and dW in 32 bits once
    return {"bytes": 2 * m * (k + n) * s + case.get("E", 1) * n * k * (s + 4), "flops": 6.0 * m * n * k}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _spread(g, rows, cols, sigma):
    """Normal values, each channel with a log-normal size of its own."""
    return _normal(g, rows, cols) * torch.exp(sigma * _normal(g, cols))


def _loads(case, seed):
    """Rows of each expert: a draw from uneven odds."""
    g = torch.Generator().manual_seed(seed * 7919 + 11)
    p = torch.softmax(case["skew"] * torch.randn(case["E"], generator=g), 0)
    got = torch.multinomial(p, case["M"], replacement=True, generator=g)
    return torch.bincount(got, minlength=case["E"])


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    st = {"case": case}
    if case["kind"] == "act":
        w = case["F"] * (2 if case["gated"] else 1)
        st["x"] = (1.5 * _spread(g, case["M"], w, 0.3)).to(dt)
        st["dh"] = (0.01 * _spread(g, case["M"], case["F"], 1.0)).to(dt)
        return st
    m, k, n, e = case["M"], case["K"], case["N"], case.get("E", 0)
    st["x"] = _spread(g, m, k, 0.5).to(dt)
    if e:
        loads = _loads(case, seed)
        st["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), loads.cumsum(0)]).to(torch.int32).to(DEVICE)
        st["capacity"] = -(-int(loads.max()) // 32) * 32
    w = (0.02 * _normal(g, *((e, n, k) if e else (n, k)))).to(dt)
    if case["kind"].endswith("train"):
        st["w"] = w
        st["dy"] = (0.001 * _spread(g, m, n, 1.0)).to(dt)
    else:
        st["w_codes"], st["w_scales"] = _packed(w)
    return st


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _scaled(x, reach):
    """(blocks of 32 of the last axis over their scales, the scales' exponents).  `reach`: what carries a significand
    into the exponent where it is past the format's range (1.75 = 7 / 4 of the 4-bit one, 127.5 / 64 of the 8-bit
    one), and the binade of the largest element."""
    over, unit = reach
    v = torch.nn.functional.pad(x.float(), (0, -x.shape[-1] % 32)).unflatten(-1, (-1, 32))
    bits = v.abs().amax(-1, keepdim=True).view(torch.int32)
    s = torch.clamp(((bits + over) >> 23) - unit, min=0)
    v = v * ((254 - s) << 23).view(torch.float32)
    return torch.where(bits < 0x7F800000, v, math.nan), s


def _scale(s):
    return torch.clamp(s << 23, min=1 << 22).view(torch.float32)    # 2^(s - 127), 2^-127 for s = 0


def _rounded4(v):
    a = v.abs()
    q = torch.where(a < 2, torch.round(2 * a) / 2, torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2)))
    return torch.copysign(torch.clamp(q, max=6.0), v)


def _mx(x):
    """The values that the 4-bit codes of `x`, in blocks along its last axis, stand for."""
    v, s = _scaled(x, (0x1FFFFF, 2))
    return (_rounded4(v) * _scale(s)).flatten(-2)[..., :x.shape[-1]]


def _act8(x):
    """The values that the 8-bit codes of `x` stand for."""
    v, s = _scaled(x, (0x10000, 6))
    return (torch.round(v) * _scale(s)).flatten(-2)[..., :x.shape[-1]]


def _packed(w):
    """A matrix (or one for each expert) as microscaled 4-bit codes in the layout of the matrix products: tiles of 16
    rows x 128 elements, in them [block of 32][row][16 bytes], two codes a byte, the earlier low; scales by 16 rows x
    512 elements, in them [block of 32 of a tile][row][tile]."""
    rows, cols = w.shape[-2:]
    v, s = _scaled(torch.nn.functional.pad(w, (0, -cols % 512, 0, -rows % 16)).reshape(-1, cols + -cols % 512), (0x1FFFFF, 2))
    q = _rounded4(v)
    a = q.abs()
    c = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
    n = c.shape[0] // 16
    b = (c[..., 0::2] | (c[..., 1::2] << 4)).view(n, 16, -1, 4, 16)
    codes = b.permute(0, 2, 3, 1, 4).contiguous()
    scales = s.to(torch.uint8).view(n, 16, -1, 4, 4).permute(0, 2, 4, 1, 3).contiguous()
    lead = w.shape[0] if w.dim() == 3 else 1
    return codes.view(lead, -1), scales.view(lead, -1)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _unpacked(codes, scales, rows, cols):
    """The values [experts, rows, cols] of _packed's codes."""
    n = -(-rows // 16)
    b = codes.view(codes.shape[0], n, -1, 4, 16, 16).permute(0, 1, 4, 2, 3, 5)
    c = torch.stack([b & 15, b >> 4], -1).long()
    v = torch.tensor(_E2M1 + tuple(-x for x in _E2M1), device=codes.device)[c].flatten(-2)
    s = scales.view(codes.shape[0], n, -1, 4, 16, 4).permute(0, 1, 4, 2, 5, 3).reshape(v.shape[:-1])
    v = v * _scale(s.to(torch.int32)).unsqueeze(-1)
    return v.reshape(codes.shape[0], n * 16, -1)[:, :rows, :cols]


def _places(offsets, m):
    """(expert, place among its rows) of every row."""
    row = torch.arange(m, device=offsets.device)
    expert = torch.bucketize(row, offsets[1:].long(), right=True)
    return expert, row - offsets.long()[expert]


def _padded(x, at, experts, capacity):
    out = torch.zeros(experts, capacity, x.shape[1], device=x.device)
    out[at] = x.float()
    return out


def _gate(p):
    """act(x) and its slope: x sigma(t) with t = x (SiLU) or 2 sqrt(2 / pi) (x + 0.044715 x^3) (GELU, tanh form)."""
    def of(x):
        if p == "silu":
            t, dt = x, 1.0
        else:
            k = 2 * math.sqrt(2 / math.pi)
            t, dt = k * (x + 0.044715 * x * x * x), k * (1 + 3 * 0.044715 * x * x)
        sg = 1 / (1 + torch.exp(-t))
        return x * sg, sg + x * sg * (1 - sg) * dt
    return of


def _plain(st):
    case, x = st["case"], st["x"]
    dt = x.dtype
    if case["kind"] == "act":
        f, act, dh = case["F"], _gate(case["act"]), st["dh"].float()
        if not case["gated"]:
            return act(x.float())[0].to(dt), (dh * act(_act8(x))[1]).to(dt)
        g, u = x[:, :f], x[:, f:]
        h = (act(g.float())[0] * u.float()).to(dt)
        g, u = _act8(g), _act8(u)
        a, slope = act(g)
        return h, torch.cat([dh * u * slope, dh * a], 1).to(dt)
    k, n = case["K"], case["N"]
    if case["kind"] == "linear":
        return (_mx(x) @ _unpacked(st["w_codes"], st["w_scales"], n, k)[0].T).to(dt)
    if case["kind"] == "linear_train":
        w, dy = st["w"], st["dy"]
        y = _mx(x) @ _mx(w).T
        dx = _mx(dy) @ _mx(w.T).T
        dw = _mx(dy.T) @ _mx(x.T).T
        return y.to(dt), dx.to(dt), dw
    at = _places(st["offsets"], case["M"])
    experts, capacity = case["E"], st["capacity"]
    if case["kind"] == "experts":
        w = _unpacked(st["w_codes"], st["w_scales"], n, k)
        return torch.bmm(_padded(_mx(x), at, experts, capacity), w.transpose(1, 2).contiguous())[at].to(dt)
    w, dy = st["w"], st["dy"]
    y = torch.bmm(_padded(_mx(x), at, experts, capacity), _mx(w).transpose(1, 2).contiguous())[at]
    dx = torch.bmm(_padded(_mx(dy), at, experts, capacity), _mx(w.transpose(1, 2)).transpose(1, 2).contiguous())[at]
    x_t = _mx(_padded(x, at, experts, capacity).transpose(1, 2))
    dy_t = _mx(_padded(dy, at, experts, capacity).transpose(1, 2))
    return y.to(dt), dx.to(dt), torch.bmm(dy_t, x_t.transpose(1, 2).contiguous())


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own(st):
    from paper_2411_10948_amd import mx

    case, x = st["case"], st["x"]
    if case["kind"] == "act":
        plan = st.get("plan")
        if plan is None:
            plan = st["plan"] = mx.ActPlan(case["M"], case["F"], case["act"], gated=case["gated"], dtype=x.dtype)
        h = plan.forward(x)
        return h, plan.backward(st["dh"])
    plan = st.get("plan")
    if plan is None:
        plan = st["plan"] = mx.LinearPlan(case["M"], case["K"], case["N"], dtype=x.dtype, experts=case.get("E", 0),
                                          train=case["kind"].endswith("train"))
    offsets = st.get("offsets")
    if not plan.train:
        w = st.get("weight")
        if w is None:
            w = st["weight"] = mx.MxMatrix(st["w_codes"], st["w_scales"], case["N"], case["K"])
        return plan.forward(x, w, offsets)
    plan.quantize_weight(st["w"])
    y = plan.forward(x, offsets=offsets)
    dx, dw = plan.backward(st["dy"])
    return y, dx, dw


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _blocks64(x, top, below):
    """Blocks of 32 of the last axis over the smallest power of two (at least 2^-127) that keeps max |x| / scale up to
    `top` (`below`: under it), and that scale."""
    v = torch.nn.functional.pad(x.double(), (0, -x.shape[-1] % 32)).unflatten(-1, (-1, 32))
    most = v.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp(most, min=2.0 ** -140) / top))
    e = torch.where(most / torch.exp2(e - 1) <= top, e - 1, e)      # log2 may be off by an ulp either way
    e = torch.where(most / torch.exp2(e) > top, e + 1, e)
    if below:
        e = torch.where(most / torch.exp2(e) == top, e + 1, e)
    scale = torch.exp2(torch.clamp(e, min=-127.0))
    return v / scale, scale


def _mx64(x):
    v, scale = _blocks64(x, 7.0, False)
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64, device=x.device)
    mid[0::2] = torch.nextafter(mid[0::2], mid[0::2] + 1)       # there a tie goes down, to the even code
    q = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)[torch.bucketize(v.abs(), mid, right=True)]
    return (torch.sign(v) * q * scale).flatten(-2)[..., :x.shape[-1]]


def _act64(x):
    v, scale = _blocks64(x, 127.5, True)
    return (torch.round(v) * scale).flatten(-2)[..., :x.shape[-1]]


def _act_and_slope64(name, x):
    if name == "silu":
        s = torch.sigmoid(x)
        return x * s, s * (1 + x * (1 - s))
    k = math.sqrt(2 / math.pi)
    th = torch.tanh(k * (x + 0.044715 * x ** 3))
    return 0.5 * x * (1 + th), 0.5 * (1 + th) + 0.5 * x * (1 - th * th) * k * (1 + 3 * 0.044715 * x * x)


def exact(case, seed):
    st = prepare(case, seed)
    x = st["x"]
    if case["kind"] == "act":
        f, dh = case["F"], st["dh"].double()
        g = x[:, :f].double()
        a, _ = _act_and_slope64(case["act"], g)
        g8, u8 = _act64(x[:, :f]), _act64(x[:, f:]) if case["gated"] else None
        a8, slope8 = _act_and_slope64(case["act"], g8)
        if not case["gated"]:
            return a, dh * slope8
        return a * x[:, f:].double(), torch.cat([dh * u8 * slope8, dh * a8], 1)
    k, n, e = case["K"], case["N"], case.get("E", 0)
    if case["kind"].endswith("train"):
        w = st["w"] if e else st["w"][None]
        w_rows, w_cols = _mx64(w), _mx64(w.transpose(1, 2)).transpose(1, 2)
    else:
        w_rows = _unpacked(st["w_codes"], st["w_scales"], n, k).double()
    xq = _mx64(x)
    cuts = st["offsets"].tolist() if e else [0, case["M"]]
    parts = [slice(lo, hi) for lo, hi in zip(cuts, cuts[1:])]
    y = torch.cat([xq[p] @ w_rows[i].T for i, p in enumerate(parts)])
    if not case["kind"].endswith("train"):
        return y
    dy = st["dy"]
    dyq = _mx64(dy)
    dx = torch.cat([dyq[p] @ w_cols[i] for i, p in enumerate(parts)])
    dw = torch.zeros(len(parts), n, k, dtype=torch.float64, device=x.device)
    for i, p in enumerate(parts):
        if p.stop > p.start:
            dw[i] = _mx64(dy[p].T) @ _mx64(x[p].T).T
    return y, dx, dw if e else dw[0]
