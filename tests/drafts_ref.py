"""Verification of drafted tokens from its definition, one request and one token at a
time in float64, for the tests of drafts.verify."""
import math


def verify_one(tokens, parents, target, draft, uniform, last):
    """One request: lists of its n tokens, parents and random numbers, rows of
    probabilities (numpy float64 [n, V]; draft or None).
    -> (path, tokens: those kept after the root and the one that follows)."""
    n, V = target.shape
    at, path = 0, [0]
    while True:
        r, z = target[at].copy(), 1.0
        for c in range(at + 1, n):
            if parents[c] != at:
                continue
            x = tokens[c]
            there = 0 <= x < V
            p = r[x] if there else 0.0
            q = 1.0 if draft is None else (draft[at][x] if there else 0.0)
            if there and uniform[c] * q * z < p:
                at = c
                path.append(c)
                break
            if draft is None:
                if there:
                    z -= r[x]
                    r[x] = 0.0
            else:
                r = (r - z * draft[at]).clip(min=0.0)
                z = math.fsum(r)
        else:
            break
    out = [tokens[i] for i in path[1:]]
    for row in (r, target[at]):
        total = math.fsum(row)
        if 0.0 < total < math.inf:
            cum = 0.0
            for j in row.nonzero()[0].tolist():
                cum += row[j]
                found = j
                if cum > last * total:
                    break
            return path, out + [found]
        if not total == 0.0:
            break
    return path, out + [-1]
