"""64-bit references of routing, the exchange by expert and low-rank adapters, and what their
results may be off.

U = 2^-24 is half a step of fp32, and a fp32 sum of values v in n steps is at most n U sum |v| off.
Each bound counts the roundings of the operator's definition in fp32 (an exponential 2 U and U
for each unit of its argument, which is rounded first; a quotient U) and half a step of the output's type.
"""
from __future__ import annotations

import torch

U = 2.0 ** -24
# half a step relative to a value, and half of the smallest number
HALF = {torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 2.0 ** -134),
        torch.float32: (2.0 ** -24, 2.0 ** -150)}


def rounded(want, off, dtype):
    """The bound of a result off by `off` before its rounding to `dtype`."""
    rel, least = HALF[dtype]
    return off + rel * (want.abs() + off) + least


def check(name, got, want, bound):
    """Every value within its bound; NaN and infinities where they are wanted.  Past the largest number
    of its type, from half a step over it, a value is infinite."""
    past = torch.finfo(got.dtype).max * (1 + torch.finfo(got.dtype).eps / 4)
    got = got.detach().double().cpu()
    assert got.shape == want.shape, f"{name}: {tuple(got.shape)}, expected {tuple(want.shape)}"
    finite = torch.isfinite(want)
    same = (got == want) | (got.isnan() & want.isnan())
    assert bool(same[~finite].all()), f"{name}: infinities or NaN differ"
    over = got.isinf() & (got.sign() == want.sign()) & (want.abs() + bound >= past)
    off = ((got - want).abs() / bound)[finite & ~over]
    assert off.numel() == 0 or bool((off <= 1).all()), \
        f"{name}: {int((~(off <= 1)).sum())} of {off.numel()} past the bound, worst {float(off.max())} of it"


# ---- routing ------------------------------------------------------------------------


def choose(logits, k, valid=None):
    """The k largest of each row: NaN above all, lower index first, -inf and rows not valid never."""
    m, experts = logits.shape
    out = torch.full((m, k), -1, dtype=torch.int32)
    for t in range(m):
        if valid is not None and not valid[t]:
            continue
        row = logits[t].tolist()
        order = sorted((e for e in range(experts) if row[e] != float("-inf")),
                       key=lambda e: (-float("inf") if row[e] != row[e] else -row[e], e))
        # NaN before +inf
        order.sort(key=lambda e: row[e] == row[e])
        for j, e in enumerate(order[:k]):
            out[t, j] = e
    return out


def route(logits, k, renormalize, valid=None):
    """(experts, weights, counts, loss, slopes) and a differentiable weights and loss, all in 64 bits
    of logits that may require a gradient."""
    m, experts = logits.shape
    chosen = choose(logits.detach(), k, valid)
    routed = chosen[:, :1].ge(0).squeeze(1)
    p = torch.zeros_like(logits)
    weights = torch.zeros((m, k), dtype=torch.float64)
    if bool(routed.any()):
        soft = torch.softmax(logits[routed], dim=1)
        p = p.index_put((routed.nonzero().squeeze(1),), soft)
        picked = torch.where(chosen >= 0, p.gather(1, chosen.clamp(min=0).long()), 0.0)
        total = picked.sum(1, keepdim=True)
        weights = torch.where(routed[:, None], picked / torch.where(routed[:, None], total, 1.0), 0.0) \
            if renormalize else picked
    counts = torch.bincount(chosen[chosen >= 0].long(), minlength=experts)
    tokens, choices = int(routed.sum()), int(counts.sum())
    slopes = experts * counts.double() / max(1, choices * tokens)
    loss = (slopes * p.sum(0)).sum()
    return chosen, weights, counts.to(torch.int32), loss, slopes


def weight_bound(logits, weights):
    """Of fp32 weights: an exponential and its argument, the sum's terms and steps, the quotient."""
    finite = torch.where(torch.isfinite(logits), logits, 0.0)
    spread = float(finite.max() - finite.min()) if logits.numel() else 0.0
    return (2 * (spread + 3) + 16 + 6 + 2) * U * weights.abs() + 2.0 ** -149


def gradient_bound(logits, weights, dweights, slopes, dloss, renormalize, chosen):
    """Of the logits' gradient before its rounding: every product's terms in absolute values, times
    the relative error of p or w and the steps of the two sums."""
    m, experts = logits.shape
    p = torch.softmax(torch.where(chosen[:, :1] >= 0, logits, 0.0), dim=1)
    finite = torch.where(torch.isfinite(logits), logits, 0.0)
    rel = (3 * (2 * (float(finite.max() - finite.min()) + 3) + 24) + 24 + 32) * U
    u = (slopes * dloss).abs().expand(m, experts).clone()
    extra = torch.zeros_like(p)
    there = (chosen >= 0).double()
    index = chosen.clamp(min=0).long()
    if renormalize:
        w = weights.abs() * there
        extra.scatter_add_(1, index, w * (dweights.abs() + (w * dweights.abs()).sum(1, keepdim=True)))
    else:
        u.scatter_add_(1, index, dweights.abs() * there)
    # the reference's own roundings, in 64 bits: where its terms cancel to 0 it has 2^-52 of them left
    own = 2.0 ** -46 * (u.sum(1, keepdim=True) + extra.sum(1, keepdim=True))
    return rel * (p * (u + (p * u).sum(1, keepdim=True)) + extra) + own + 2.0 ** -140


# ---- exchange -----------------------------------------------------------------------


def group(ids, groups):
    """(ends, rows, slots) by going through the slots."""
    flat = ids.reshape(-1).tolist()
    bins = [[s for s, g in enumerate(flat) if g == e] for e in range(groups)]
    rest = [s for s, g in enumerate(flat) if not 0 <= g < groups]
    slots = [s for b in bins for s in b]
    rows = torch.full((len(flat),), -1, dtype=torch.int32)
    if slots:
        rows[torch.tensor(slots)] = torch.arange(len(slots), dtype=torch.int32)
    ends = torch.tensor([len(b) for b in bins], dtype=torch.int64).cumsum(0).to(torch.int32)
    return ends, rows.view(ids.shape), torch.tensor(slots + rest, dtype=torch.int32)


def dispatch(x, rows, places):
    out = torch.zeros((places, x.shape[1]), dtype=x.dtype)
    for t, r in enumerate(rows.reshape(x.shape[0], -1).tolist()):
        for place in r:
            if place >= 0:
                out[place] = x[t]
    return out


def combine(y, rows, weights=None):
    """(out, sum of absolute values): 64 bits."""
    keep = (rows >= 0) & (rows < y.shape[0])
    picked = torch.where(keep[..., None], y.double()[torch.where(keep, rows, 0).long()], 0.0) \
        if y.shape[0] else torch.zeros((*rows.shape, y.shape[1]), dtype=torch.float64)
    if weights is not None:
        picked = torch.where(keep[..., None], picked * weights.double()[..., None], 0.0)
    return picked.sum(1), picked.abs().sum(1)


# ---- adapters -----------------------------------------------------------------------


def groups_of(ends, m):
    return [(0, m)] if ends is None else list(zip([0, *ends.tolist()[:-1]], ends.tolist()))


def adapt(x, down, up, ends, slots, y, scales, parts_off, floor):
    """(out, bound before the rounding, h by place, h's bound) in 64 bits.

    `parts_off`: what the parts of h leave of it, relative; `floor`: relative to the row's largest."""
    m, n, rank, k = x.shape[0], up.shape[2], down.shape[1], x.shape[1]
    out = torch.zeros((m, n), dtype=torch.float64) if y is None else y.double().clone()
    off = torch.zeros_like(out)
    h = torch.zeros((m, rank), dtype=torch.float64)
    h_off = torch.zeros_like(h)
    order = torch.arange(m) if slots is None else slots.long()
    for g, (low, high) in enumerate(groups_of(ends, m)):
        t = order[low:high]
        s = 1.0 if scales is None else float(scales[g])
        xd, dd, ud = x[t].double(), down[g].double(), up[g].double()
        h[low:high] = xd @ dd.t()
        # steps of the sum over k: those of a matrix instruction, four waves and up to 16 shares
        h_off[low:high] = (k / 32 + 32 + 4 + 16) * U * (xd.abs() @ dd.abs().t())
        delta = s * (h[low:high] @ ud)
        size = abs(s) * (h[low:high].abs() @ ud.abs())
        most = h[low:high].abs().amax(1, keepdim=True) if rank else 0.0
        off[t] = abs(s) * (h_off[low:high] @ ud.abs()) + (parts_off + (rank / 32 + 32 + 3) * U) * size \
            + floor * abs(s) * most * ud.abs().sum(0) + U * (out[t] + delta).abs()
        out[t] += delta
    return out, off, h, h_off


def parts(dtype, out):
    """What the parts of h leave of it: (relative, relative to the row's largest)."""
    if dtype is torch.float16:
        return 2.0 ** -22, 2.0 ** -34
    return (2.0 ** -23 if out is torch.float32 else 2.0 ** -16), 0.0


def weight_gradient(h, x, ends, slots, scales, dtype, out):
    """(gradient, bound before the rounding) in 64 bits."""
    m, rank, width = x.shape[0], h.shape[1], x.shape[1]
    spans = groups_of(ends, m)
    want = torch.zeros((len(spans), rank, width), dtype=torch.float64)
    off = torch.zeros_like(want)
    order = torch.arange(m) if slots is None else slots.long()
    rel, floor = parts(dtype, out)
    for g, (low, high) in enumerate(spans):
        if low >= high:
            continue
        s = 1.0 if scales is None else float(scales[g])
        xd, hd = x[order[low:high]].double(), h[low:high].double()
        want[g] = s * (hd.t() @ xd)
        steps = (high - low) / 32 + 32 + 8 + 16 + 2
        off[g] = abs(s) * ((rel + steps * U) * (hd.abs().t() @ xd.abs())
                           + floor * hd.abs().max() * xd.abs().sum(0))
    return want, off
