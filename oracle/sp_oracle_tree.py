"""CPU oracle for several tokens a step: tree attention over the joined cache, sampling, acceptance (TEST INFRASTRUCTURE ONLY).

Plain, slow numpy in fp64, written from the definitions in include/sp.h, sharing no code with the HIP path.

  tree_attention   one prompt: node i sees every cached key and, of the tree, its ancestors and itself
  sample_row       one row of logits: the tokens in order, the three filters one after the other, the draw
  accept_walk      one prompt: the nodes that the walk takes and what was sampled at the last of them
"""
from __future__ import annotations

import math

import numpy as np


def lineage(parent, i):
    """Node i's ancestors from the root down, then i."""
    out = []
    while i >= 0:
        out.append(i)
        up = int(parent[i])
        i = up if 0 <= up < i else -1
    return out[::-1]


def tree_attention(q, k_new, v_new, k_old, v_old, parent, scale, slopes=None, pos_q=None, pos_old=None):
    """q [n, Hq, d]; k_new, v_new [n, Hkv, d]; k_old, v_old [S, Hkv, d].  Returns (o [n, Hq, d], sum of weight * |v| likewise,
    largest scale * sum |q k| (+ |penalty|) of any key: what rounding errors are measured by)."""
    q, k_new, v_new, k_old, v_old = (np.asarray(a, np.float64) for a in (q, k_new, v_new, k_old, v_old))
    n, Hq, d = q.shape
    G = Hq // k_new.shape[1]
    o, absum, big = np.zeros((n, Hq, d)), np.zeros((n, Hq, d)), np.zeros((n, Hq))
    for i in range(n):
        line = lineage(parent, i)
        for h in range(Hq):
            K = np.concatenate([k_old[:, h // G], k_new[line, h // G]])
            V = np.concatenate([v_old[:, h // G], v_new[line, h // G]])
            s = scale * (K @ q[i, h])
            size = scale * (np.abs(K) @ np.abs(q[i, h]))
            if slopes is not None:
                away = pos_q[i] - np.concatenate([np.asarray(pos_old, np.float64), np.asarray(pos_q, np.float64)[line]])
                s = s - slopes[h] * away
                size = size + slopes[h] * np.abs(away)
            a = np.exp(s - s.max())
            a /= a.sum()
            o[i, h], absum[i, h], big[i, h] = a @ V, a @ np.abs(V), size.max()
    return o, absum, big


def sample_order(x):
    """Indices of the logits that take part, in order: descending, ties by the lower index."""
    x = np.asarray(x, np.float64)
    live = np.flatnonzero(~np.isnan(x) & (x != -np.inf))
    return live[np.argsort(-x[live], kind="stable")]


def sample_weights(x, order, temperature):
    x = np.asarray(x, np.float64)
    m = x[order[0]]
    if np.isinf(m):
        return (x[order] == m).astype(np.float64)
    return np.exp((x[order] - m) / float(temperature))


def sample_row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, margin): margin is the smallest relative distance of any decision (min-p, top-p, draw) from its border."""
    order = sample_order(x)
    if len(order) == 0:
        return -1, -np.inf, np.inf
    if not temperature > 0:
        return int(order[0]), 0.0, np.inf
    w = sample_weights(x, order, temperature)
    margin = np.inf
    if min_p > 0:
        limit = min(float(min_p), 1.0)
        off = np.abs(w / limit - 1)
        margin = min(margin, float(off[off > 0].min()) if (off > 0).any() else np.inf)
        w = w[w >= limit]
    if top_k > 0:
        w = w[:top_k]
    run = np.cumsum(w)
    if top_p < 1:
        border = max(float(top_p), 0.0) * run[-1]
        kept = max(1, int((run - w < border).sum()))
        near = np.abs((run - border) / run[-1])
        margin = min(margin, float(near[:-1].min()) if len(near) > 1 else np.inf)
        w, run = w[:kept], run[:kept]
    if not u >= 0:
        u = 0.0
    u = min(float(u), 1.0 - 2.0 ** -24)
    j = min(int((run <= u * run[-1]).sum()), len(w) - 1)
    margin = min(margin, float(np.abs(run - u * run[-1]).min() / run[-1]) if u > 0 else margin)
    return int(order[j]), math.log(w[j]) - math.log(run[-1]), margin


def accept_walk(parent, n, draft, sampled, room):
    """Nodes that are taken, what was sampled at the last (-1: no node).  room: nodes that found a place in the cache."""
    n = min(n, room)
    if n <= 0:
        return [], -1
    path = [0]
    while True:
        drawn = int(sampled[path[-1]])
        child = [i for i in range(path[-1] + 1, n) if int(parent[i]) == path[-1] and int(draft[i]) == drawn and drawn >= 0]
        if not child:
            return path, drawn
        path.append(child[0])
