"""CPU oracle for drafted trees over the tiered cache (test infrastructure, like tkv_oracle.py): attention of a tree, the walk
against the target's probabilities, the path that is kept.  float64 throughout.  Pins: tests/test_tree_oracle.py (a line of nodes is a
chunk of tokens; the walk's tokens are distributed as the target's; hand-worked walks)."""
from __future__ import annotations

import numpy as np

from .tkv_oracle import T0, T3, OracleCache, attend_gqa


def ancestors(parents: np.ndarray):
    """For parents [n]: for every node the ascending list of its ancestors and itself, or None where it is not there (a parent
    outside -1 .. i - 1, its own or an ancestor's)."""
    lines = []
    for i, p in enumerate(np.asarray(parents, dtype=np.int64)):
        if p == -1:
            lines.append([i])
        elif 0 <= p < i and lines[p] is not None:
            lines.append(lines[p] + [i])
        else:
            lines.append(None)
    return lines


def walk(parents, tokens, p, q, u_accept, u_draw):
    """One sequence: parents, tokens, u_accept [n], p, q [n, vocab] (q None: children chosen by rank).  Returns (path, next token)."""
    n = len(parents)
    p = np.asarray(p, dtype=np.float64)
    q = None if q is None else np.asarray(q, dtype=np.float64)
    cur, path, t, total = 0, [0], p[0].copy(), 1.0
    i = 1
    while i < n:
        if parents[i] == cur:
            x = int(tokens[i])
            inside = 0 <= x < p.shape[1]
            left = t[x] if inside else 0.0
            drafted = 1.0 if q is None else (q[cur, x] if inside else 0.0)
            if float(u_accept[i]) * total * drafted < left:
                cur, t, total = i, p[i].copy(), 1.0
                path.append(i)
            else:
                r = t.copy() if q is None else np.maximum(t - total * q[cur], 0.0)
                if q is None and inside:
                    r[x] = 0.0
                mass = total - left if q is None else r.sum()
                if mass > 0.0:
                    t, total = r, mass
        i += 1
    run = np.cumsum(t)
    above = np.nonzero(run > float(u_draw) * run[-1])[0]
    return path, int(above[0]) if len(above) else p.shape[1] - 1


class TreeOracleCache(OracleCache):
    """OracleCache with trees.  The nodes' rows are the last n positions of every layer."""

    def __init__(self, *a, **kw):
        super().__init__(*a, **kw)
        self.tree_weights = {}

    def attend_tree(self, layer, q, parents):
        """q [B, n, Hq, d], parents [B, n].  Returns out [B, n, Hq, d]; keeps the weights for accept_tree."""
        q = np.asarray(q, dtype=np.float64)
        B, n = q.shape[:2]
        N = self.length[layer]
        base = N - n
        out = np.zeros(q.shape)
        weights = np.zeros((B, n, self.Hq, N))
        for b in range(B):
            for i, line in enumerate(ancestors(parents[b])):
                if line is None:
                    continue
                live = np.zeros((1, N), dtype=bool)
                live[0, :base] = self.tier[b, :base] != T3
                live[0, [base + j for j in line]] = True
                o, w = attend_gqa(q[b:b + 1, i], self.K[layer][b:b + 1, :, :N] * live[:, None, :, None],
                                  np.where(live[:, None, :, None], self.V[layer][b:b + 1, :, :N], 0.0), live, self.softmax_scale)
                out[b, i], weights[b, i] = o[0], w[0]
        self.tree_weights[layer] = weights
        return out

    def accept_tree(self, n, paths, scored=True):
        """paths: per sequence the list of kept nodes, ascending."""
        N = self.length[self.layers[0]]
        base = N - n
        keep = max(len(p) for p in paths)
        for b, path in enumerate(paths):
            if scored:
                for l in self.layers:
                    w = self.tree_weights[l][b, path]                                   # [kept, Hq, N]
                    if self.scorer == "vatp":
                        w = w * np.repeat(self.vnorm[l][b, :, :N], self.G, 0)[None]
                    self.score[b, :N] += self.score_scale * w.sum((0, 1))
            at = [base + i for i in path]
            for l in self.layers:
                arrays = [self.K[l][b], self.V[l][b]] + ([self.vnorm[l][b]] if self.vnorm is not None else [])
                for x in arrays:
                    rows = x[:, at].copy()
                    x[:, base:N] = 0.0
                    x[:, base:base + len(path)] = rows
            kept = self.score[b, at].copy()
            self.score[b, base:N] = 0.0
            self.score[b, base:base + len(path)] = kept
            self.tier[b, base:N] = T0
            self.tier[b, base + len(path):base + keep] = T3
        for l in self.layers:
            self.length[l] = base + keep
        self.tree_weights = {}
        return keep

    def classify(self, policy_ppm, score_f32=None, count_rule=0):
        new = super().classify(policy_ppm, score_f32, count_rule)
        new[self.tier == T3] = T3                # a node that was not kept stays evicted where the window protects the others
        return new
