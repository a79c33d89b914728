"""CPU oracle for the operators on rows of vocabulary logits.  TEST INFRASTRUCTURE ONLY.

Same rules as specs_oracle.py: float64 numpy and plain Python loops, the definitions of include/specs.h written out,
nothing imported from the product, never called by it.

  sample       one token per row from a given uniform: temperature, top-k, top-p and min-p in this order on the entries
               sorted by (logit descending, id ascending), whole-number weights rint(2^31 exp((l - max) / T))
  top_logits   the K largest logits and the log-sum-exp at a temperature
  distill      divergence of the student's softmax from a teacher's list, and its gradient
"""
from __future__ import annotations

import math

import numpy as np


def _in_order(x):
    """Ids of the entries above -inf (and no NaN): larger logit first, lower id first among equals."""
    ids = np.nonzero(x > -math.inf)[0]
    return [int(i) for i in ids[np.argsort(-x[ids], kind="stable")]]


def sample(logits, uniforms, temperature=None, top_k=None, top_p=None, min_p=None):
    """Per row a dict: token, logprob, draw_logprob, ``margin`` -- how far, relative to the mass, the decisions are from
    turning out otherwise (nucleus boundary and draw) -- ``near``: the tokens of the sorted entries next to the drawn
    one, and ``low_margin``: how far min_p's bound on z is from the nearest entry."""
    out = []
    for r in range(len(logits)):
        x = np.asarray(logits[r], dtype=np.float64)
        t = 1.0 if temperature is None else float(np.float32(temperature[r]))
        u = float(np.float32(uniforms[r]))
        u = min(max(u, 0.0), 1.0 - 2.0**-24)
        order = _in_order(x)
        if not len(order):
            out.append(dict(token=-1, logprob=math.nan, draw_logprob=math.nan, margin=math.inf, near=[-1], low_margin=math.inf))
            continue
        k = 0 if top_k is None else int(top_k[r])
        m = x[order[0]]
        if not t > 0 or m == math.inf:
            t, k = 1.0, 1
        with np.errstate(over="ignore", invalid="ignore"):
            z = np.array([0.0 if x[i] == m else (x[i] - m) / t for i in order])
            w = np.rint(np.exp(z) * 2.0**31)
            ln_sum = math.nan if np.isnan(x).any() or m == math.inf else math.log(np.exp(x - m).sum())
        n = len(order)
        if k > 0:
            n = min(n, k)
        total = w[:n].sum()
        margin, low_margin = math.inf, math.inf
        before = np.concatenate([[0.0], np.cumsum(w)])
        p = 1.0 if top_p is None else float(np.float32(top_p[r]))
        if p < 1:
            goal = math.floor(total * p)
            margin = min(margin, float(np.abs(before[1:n] - goal).min(initial=math.inf)) / total)
            n = max(1, int(np.sum(before[:n] < goal)))
        q = 0.0 if min_p is None else float(np.float32(min_p[r]))
        if q > 0:
            low = math.log(min(q, 1.0))
            away = np.abs(z - low)
            low_margin = float(away[z != 0.0].min(initial=math.inf))   # the largest entries themselves are exact
            n = min(n, int(np.sum(z >= low)))
        kept = before[n]
        goal = math.floor(kept * u)
        at = int(np.searchsorted(before[1:n + 1], goal, side="right"))
        inner = before[1:n]
        margin = min(margin, float(np.abs(inner - goal).min(initial=math.inf)) / kept)
        near = [order[i] for i in range(max(0, at - 1), min(n, at + 2))]
        out.append(dict(token=order[at], logprob=x[order[at]] - m - ln_sum, draw_logprob=z[at] - math.log(kept * 2.0**-31),
                        margin=margin, near=near, low_margin=low_margin))
    return out


def top_logits(logits, K, temperature=1.0):
    """ids [rows, K], values [rows, K] (padded with -1 / -inf), lse [rows]."""
    rows = len(logits)
    ids, values, lse = np.full((rows, K), -1, np.int32), np.full((rows, K), -math.inf), np.zeros(rows)
    for r in range(rows):
        x = np.asarray(logits[r], dtype=np.float64)
        order = _in_order(x)[:K]
        ids[r, :len(order)], values[r, :len(order)] = order, x[order]
        if np.isnan(x).any() or (x == math.inf).any():
            lse[r] = math.nan
        elif not len(order):
            lse[r] = -math.inf
        else:
            z = x / temperature
            lse[r] = z.max() + math.log(np.exp(z - z.max()).sum())
    return ids, values, lse


def distill(logits, top_ids, top_values, temperature=1.0, top_lse=None, row_weight=None, grad_loss=None):
    """loss [rows], stats [rows, 3], grad [rows, V], and the pieces a tolerance is made of (p, q, q_r / p_r per row)."""
    logits = np.asarray(logits, dtype=np.float64)
    rows, V = logits.shape
    T = float(np.float32(temperature))
    loss, stats, grad = np.zeros(rows), np.zeros((rows, 3)), np.zeros((rows, V))
    p_all, q_all, ratio = np.zeros((rows, V)), np.zeros((rows, V)), np.zeros(rows)
    for r in range(rows):
        weight = 1.0 if row_weight is None else float(np.float32(row_weight[r]))
        if weight == 0:
            continue
        here = [(int(i), float(t)) for i, t in zip(top_ids[r], top_values[r]) if i >= 0]
        if any(i >= V for i, _ in here):
            loss[r] = math.nan
            continue
        t = np.array([t for _, t in here]) / T
        if top_lse is not None:
            ref, ln_mass = float(np.float32(top_lse[r])), 0.0
        else:
            # (never added up: next to a lowest value the logarithm would be lost)
            ref = t.max() if len(t) and t.max() > -math.inf else 0.0
            mass = np.exp(t - ref).sum()
            ln_mass = math.log(mass) if mass > 0 else math.inf
        q = np.exp((t - ref) - ln_mass) if len(t) else np.zeros(0)
        x = logits[r]
        top = float(np.nanmax(x)) if not np.isnan(x).all() else -math.inf
        with np.errstate(invalid="ignore", divide="ignore"):
            e = np.exp((x - (top if top > -math.inf else 0.0)) / T)
            listed = np.zeros(V, dtype=bool)
            listed[[i for i, _ in here]] = True
            total, rest = e.sum(), e[~listed].sum()
            q_r = max(0.0, 1.0 - q.sum()) if top_lse is not None and not rest == 0 else 0.0
            if q_r > 0 and not np.isnan(rest) and (top - float(np.nanmax(x[~listed]))) / T > 690:   # what lies further down counts as nothing
                q_r = 0.0
            S = q.sum() + q_r
            value = 0.0
            for (i, _), qj in zip(here, q):
                if qj != 0:
                    value += qj * (math.log(qj) - ((x[i] - top) / T - math.log(total) if total > 0 and x[i] > -math.inf else
                                                   (math.nan if np.isnan(total) else -math.inf)))
            if q_r > 0:
                value += q_r * (math.log(q_r) - math.log(rest / total))
                ratio[r] = q_r * total / rest
            p = e / total if not total == 0 else np.zeros(V)
        loss[r] = weight * value
        stats[r] = (top, total, rest if top_lse is not None else 0.0)
        g = p * np.where(listed, S, S - ratio[r])
        for (i, _), qj in zip(here, q):
            g[i] -= qj
            q_all[r, i] += qj
        p_all[r] = p
        grad[r] = g * weight * (1.0 if grad_loss is None else float(np.float32(grad_loss[r]))) / T
    return loss, stats, grad, dict(p=p_all, q=q_all, ratio=ratio)
