"""Plain forms of what comes before and after a step's attention (CPU, loops over requests and tokens): the table of pages and the batch's rows, and the draw
of a token from logits in binary64."""
import math

import numpy as np
import torch


def plan_ref(page, num_pages, max_pages, pages, held, free, free_count, cached, fresh, tokens, fixed=None):
    """The step, one request after the other.  Lists in (copied), a dict of lists out."""
    pages, held, free = [list(r) for r in pages], [min(max(h, 0), max_pages) for h in held], list(free)
    cached, fresh = [max(c, 0) for c in cached], [max(f, 0) for f in fresh]
    R, count = len(held), min(max(free_count, 0), num_pages)
    fixed = [min(max(f, 0), h) for f, h in zip(fixed, held)] if fixed is not None else [0] * R
    start = [0]
    for f in fresh:
        start.append(start[-1] + f)
    need = [-(-(cached[r] + fresh[r]) // page) for r in range(R)]
    lack = [-1 if need[r] > max_pages or start[r + 1] > tokens else 0 for r in range(R)]
    want = [held[r] if lack[r] else max(need[r], fixed[r]) for r in range(R)]
    for r in range(R):
        for j in range(want[r], held[r]):
            free[count] = pages[r][j]
            count += 1
        held[r] = min(held[r], want[r])
    out_of_pages = False
    for r in range(R):
        n = want[r] - held[r]
        if n == 0:
            continue
        if n > count or out_of_pages:
            lack[r], out_of_pages = n, True
            continue
        for j in range(held[r], want[r]):
            count -= 1
            pages[r][j] = free[count]
        held[r] = want[r]
    positions, slots, owner = [0] * tokens, [-1] * tokens, [-1] * tokens
    for r in range(R):
        for t in range(start[r], min(start[r + 1], tokens)):
            p = cached[r] + t - start[r]
            positions[t], owner[t] = p, r
            if lack[r] == 0 and 0 <= pages[r][p // page] < num_pages:
                slots[t] = pages[r][p // page] * page + p % page
    return {"q_start": [min(s, tokens) for s in start], "kv_len": [0 if lack[r] else cached[r] + fresh[r] for r in range(R)], "lack": lack, "held": held,
            "free_count": [count], "positions": positions, "slots": slots, "owner": owner, "pages": pages, "free": free}


# How near to a border a draw may be for the two sides' sums to put it on different sides: both sum at most 2^22 weights of binary64, each off by a few units
# of its last place, in some order.
NEAR = 2.0 ** -53 * 2 ** 22


def sample_ref(logits, temperature, top_k, top_p, min_p, u):
    """(token, probability, near) of one row, tokens sorted one by one.  near: a border of top-p, min-p or the draw is nearer than the sums are sure of."""
    x = logits.double().cpu().numpy() + 0.0
    x = np.where(np.isnan(x), -np.inf, x)
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if order.size == 0:
        return -1, 0.0, False
    if not temperature > 0 or top_k == 1:
        return int(order[0]), 1.0, False
    v = x[order]
    with np.errstate(invalid="ignore"):
        d = np.where(v == v[0], 0.0, v - v[0])
    w = np.exp(d / temperature)
    near = False
    if 0 < top_k < w.size:
        w = w[:top_k]
    if top_p < 1:
        before, goal = np.cumsum(w) - w, top_p * math.fsum(w)
        near |= bool(np.any((np.abs(before[1:] - goal) < NEAR * goal) & (w[1:] > 0) & (before[1:] != goal)))
        w = w[: max(1, int((before < goal).sum()))]
    if min_p > 0:
        least = min(min_p, 1.0)
        near |= bool(np.any((np.abs(w - least) < 1e-14) & (w != least)))
        w = w[: int((w >= least).sum())]
    total = math.fsum(w)
    upto, goal = np.cumsum(w), min(max(u, 0.0), 1 - 2.0 ** -24) * total
    near |= bool(np.any((np.abs(upto[:-1] - goal) < NEAR * total) & (upto[:-1] != goal)))
    i = min(int((upto <= goal).sum()), w.size - 1)
    return int(order[i]), float(w[i] / total), near


def assert_drawn(token, probability, logits, temperature, top_k, top_p, min_p, uniform, what=""):
    """Every row's token is the reference's (unless a border is too near to say) and its probability is off by no more than its rounding and the sums'."""
    unsure = 0
    for r in range(logits.shape[0]):
        ref, p, near = sample_ref(logits[r], float(temperature[r]), int(top_k[r]) if top_k is not None else 0, float(top_p[r]) if top_p is not None else 1.0,
                                  float(min_p[r]) if min_p is not None else 0.0, float(uniform[r]))
        if near:
            unsure += 1
            continue
        assert int(token[r]) == ref, (what, r, int(token[r]), ref, float(probability[r]), p)
        assert abs(float(probability[r]) - p) <= (2.0 ** -24 + 2 * NEAR) * p, (what, r, float(probability[r]), p)
    return unsure
