"""Plain 64-bit forms of the operators of a layer with experts, one token, pair or expert at a time, written from their definitions."""
import math

import torch


def scores(l, score):
    """[T, E] in float64; closed experts have 0."""
    closed = l == -math.inf
    if score == "sigmoid":
        return torch.where(closed, 0.0, 1 / (1 + torch.exp(-l)))
    top = l.amax(1, keepdim=True)
    e = torch.where(closed, 0.0, torch.exp(l - torch.where(top == -math.inf, 0.0, top)))
    total = e.sum(1, keepdim=True)
    return e / torch.where(total == 0, 1.0, total)


def choose(l, k, score, bias, groups, keep, best):
    """Experts [T, k], by going through each token's on the host: Python's sort is stable, so that of equals the first comes first."""
    s = scores(l, score)
    c = l if bias is None and groups == 1 else torch.where(l == -math.inf, -math.inf, s if bias is None else s + bias)
    number = lambda v: (v == v, v if v == v else 0.0)  # noqa: E731  NaN comes after everything
    per, out = l.shape[1] // groups, []
    for row in c.tolist():
        ids = list(range(groups))
        of = lambda g: sum(sorted(row[g * per: (g + 1) * per], key=number, reverse=True)[:best])  # noqa: B023, E731
        ids = sorted(ids, key=lambda g: number(of(g)), reverse=True)[:keep] if groups > 1 else ids
        open_ = sorted(e for g in ids for e in range(g * per, (g + 1) * per))
        out.append(sorted(open_, key=lambda e: number(row[e]), reverse=True)[:k])  # noqa: B023
    return torch.tensor(out, dtype=torch.int64).reshape(l.shape[0], k)


def weights(l, experts, score, renormalize, scale):
    """[T, k] from logits [T, E] that may require gradients; a token whose chosen experts are all closed has zeros."""
    closed = l == -math.inf
    if renormalize:
        chosen = torch.gather(l if score == "softmax" else torch.nn.functional.logsigmoid(l), 1, experts)
        none = (chosen == -math.inf).all(1, keepdim=True)
        return torch.where(none, 0.0, torch.softmax(torch.where(none, 0.0, chosen), 1)) * scale
    if score == "sigmoid":
        return torch.gather(torch.sigmoid(l), 1, experts) * scale
    none = closed.all(1, keepdim=True)
    return torch.gather(torch.where(none, 0.0, torch.softmax(torch.where(none, 0.0, l), 1)), 1, experts) * scale


def in_order(experts, E, first=0):
    """(offsets, rows, place) as lists."""
    e = experts.reshape(-1).tolist()
    rows = [i for x in range(first, first + E) for i, v in enumerate(e) if v == x]
    offsets = [0]
    for x in range(first, first + E):
        offsets.append(offsets[-1] + sum(v == x for v in e))
    place = [-1] * len(e)
    for r, i in enumerate(rows):
        place[i] = r
    return offsets, rows + [-1] * (len(e) - len(rows)), place
