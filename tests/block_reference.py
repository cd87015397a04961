"""Plain implementation in 64 bits of layer norm, the router and the exchange of
rows, from the definitions in include/shiftquant.h.  Test infrastructure only
(numpy, no library code)."""
import itertools
import math

import numpy as np

U = 2.0 ** -24      # half a step of fp32, relative


def norm(h, gamma, beta, eps):
    """(y, xh, r)"""
    mean = h.mean(1, keepdims=True)
    r = 1.0 / np.sqrt(((h - mean) ** 2).mean(1, keepdims=True) + eps)
    xh = (h - mean) * r
    return xh * gamma + beta, xh, r


def norm_backward(h, gamma, eps, dy, dh=0.0):
    """(dx, dgamma, dbeta)"""
    _, xh, r = norm(h, gamma, 0.0, eps)
    q = dy * gamma
    dx = r * (q - q.mean(1, keepdims=True) - xh * (q * xh).mean(1, keepdims=True)) + dh
    return dx, (dy * xh).sum(0), dy.sum(0)


def scores(logits, score):
    with np.errstate(over="ignore"):
        if score == "sigmoid":
            return 1.0 / (1.0 + np.exp(-logits))
        top = logits.max()
        if top == -np.inf:
            return np.zeros_like(logits)
        x = np.exp(logits - top)
        return x / x.sum()


def group_totals(l, value, s, bias, groups):
    """Sum of a group's two highest s (+ bias), -inf where none can be chosen."""
    per, total = len(l) // groups, []
    for g in range(groups):
        best = [e for e in sorted(range(g * per, (g + 1) * per), key=lambda e: (-value[e], e))
                if l[e] > -np.inf and value[e] > -np.inf][:2]
        # rounded once, so that sums of the same scores and biases are equal however these are paired
        terms = list(s[best]) + ([] if bias is None else list(bias[best]))
        total.append(math.fsum(terms) if best else -np.inf)
    return total


def kept_groups(total, top_groups, slack=0.0):
    """Every choice of groups where totals that are `slack` apart may come in either order (0: the one choice)."""
    order = sorted(range(len(total)), key=lambda g: (-total[g], g))
    if slack == 0.0:
        return [order[:top_groups]]
    edge = total[order[top_groups - 1]]
    sure = [g for g in order if total[g] > edge + slack]
    tied = [g for g in order if abs(total[g] - edge) <= slack]
    return [sure + list(c) for c in itertools.combinations(tied, top_groups - len(sure))]


def choices(l, k, score, bias, groups, top_groups, slack=0.0):
    """(the experts of a token for every choice of groups, whether the token has shares at all)"""
    live = ~(l == -np.inf)
    s = scores(l, score) if not np.isnan(l).any() else l
    value = s + (0.0 if bias is None else bias)
    if np.isnan(l).any() or np.isnan(value[live]).any() or (score == "softmax" and (l == np.inf).any()):
        return [[]], False
    key, out = np.where(live, l if bias is None else value, -np.inf), []
    for kept in kept_groups(group_totals(l, value, s, bias, groups), top_groups, slack) if groups > 1 else [[0]]:
        mine = np.where(np.isin(np.arange(len(l)) // (len(l) // groups), kept), key, -np.inf)
        out.append([e for e in sorted(range(len(l)), key=lambda e: (-mine[e], e)) if mine[e] > -np.inf][:k])
    return out, True


def places(chosen, E):
    """(place, offsets) of a stable sort by expert"""
    flat = chosen.reshape(-1)
    place, offsets = np.full(flat.shape, -1), [0]
    for e in range(E):
        mine = np.flatnonzero(flat == e)
        place[mine] = offsets[-1] + np.arange(len(mine))
        offsets.append(offsets[-1] + len(mine))
    return place.reshape(chosen.shape), np.array(offsets)


def route(logits, k, score="softmax", bias=None, groups=1, top_groups=1, renormalize=False, scale=1.0, like=None, slack=0.0):
    """(share, chosen, place, offsets), a token and an expert at a time.  like: chosen experts to take where group totals
    that are `slack` apart allow them."""
    T, E = logits.shape
    share, chosen = np.zeros((T, k)), np.full((T, k), -1)
    for t in range(T):
        one, fine = choices(logits[t], k, score, bias, groups, top_groups)
        if not fine:
            share[t] = np.nan
            continue
        order = one[0]
        if like is not None and list(like[t][like[t] >= 0]) != order:
            other = [o for o in choices(logits[t], k, score, bias, groups, top_groups, slack)[0] if o == list(like[t][like[t] >= 0])]
            order = (other or one)[0]
        s = scores(logits[t], score)[order]
        chosen[t, :len(order)] = order
        share[t, :len(order)] = scale * (s / max(s.sum(), 1e-300) if renormalize else s)
    return (share, chosen, *places(chosen, E))


def shares(logits, chosen, score, renormalize, scale):
    """The shares of a given choice, the function that the router's gradient is of."""
    out = np.zeros(chosen.shape)
    for t, row in enumerate(chosen):
        at = row[row >= 0]
        s = scores(logits[t], score)[at]
        out[t, :len(at)] = scale * (s / max(s.sum(), 1e-300) if renormalize else s)
    return out


def route_backward(logits, chosen, dshare, score, renormalize, scale):
    """(gradient of the logits, sum of the magnitudes of its terms)"""
    grad, mag = np.zeros_like(logits), np.zeros_like(logits)
    for t, row in enumerate(chosen):
        at = row[row >= 0]
        s, d = scores(logits[t], score), dshare[t, :len(at)]
        if renormalize:
            r = s[at] / max(s[at].sum(), 1e-300)
            g, m = scale * r * (d - (d * r).sum()), abs(scale) * r * (np.abs(d) + (np.abs(d) * r).sum())
            if score == "sigmoid":
                g, m = g * (1 - s[at]), m * (1 - s[at])
            grad[t, at], mag[t, at] = g, m
        elif score == "sigmoid":
            grad[t, at] = scale * d * s[at] * (1 - s[at])
            mag[t, at] = np.abs(grad[t, at])
        else:
            of = np.zeros(len(s))
            of[at] = d
            grad[t] = scale * s * (of - (of * s).sum())
            mag[t] = abs(scale) * s * (np.abs(of) + (np.abs(of) * s).sum())
    return grad, mag


def dispatch(x, place, rows):
    t, j = np.nonzero((place >= 0) & (place < len(rows)))
    rows[place[t, j]] = x[t]
    return rows


def combine(rows, place, share, add=0.0):
    """(sums, sums of the magnitudes)"""
    some = (place >= 0) & (place < len(rows))
    terms = rows[np.where(some, place, 0)] * np.where(some, 1.0 if share is None else share, 0.0)[..., None]
    terms = np.where(some[..., None], terms, 0.0)
    return terms.sum(1) + add, np.abs(terms).sum(1) + np.abs(add)


def combine_backward(dout, rows, place, share, drows):
    some = (place >= 0) & (place < len(rows))
    for t, j in zip(*np.nonzero(some)):
        drows[place[t, j]] = share[t, j] * dout[t]
    terms = np.where(some[..., None], dout[:, None] * rows[np.where(some, place, 0)], 0.0)
    return drows, terms.sum(2), np.abs(terms).sum(2)
