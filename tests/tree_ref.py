"""Plain forms in 64 bits for the tests of drafted rows: who sees whom, attention under such a mask, the walk along agreed tokens."""
import math

import torch


def seen(parent, n):
    """[n, n] truth values: row i sees row j.  parent None: a chain; a value outside 0 .. i-1 is no parent."""
    s = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        s[i, i] = True
        up = i - 1 if parent is None else int(parent[i])
        if 0 <= up < i:
            s[i] |= s[up]
    return s


def attend(q, k, v, sees, sm_scale):
    """(out, lse, sum of weights times |v|, largest sum of |q_c k_c| * sm_scale): q [n, Hq, hd], k, v [L, Hkv, hd] in fp64, sees [n, L]."""
    n, Hq, hd = q.shape
    rep = Hq // k.shape[1]
    out, lse, spread = torch.zeros_like(q), torch.full((n, Hq), -math.inf, dtype=torch.float64), torch.zeros_like(q)
    terms = 0.0
    for h in range(Hq):
        kk, vv = k[:, h // rep], v[:, h // rep]
        s = (q[:, h] @ kk.T) * sm_scale
        terms = max(terms, float((q[:, h].abs() @ kk.abs().T).max()) * sm_scale)
        s[~sees] = -math.inf
        lse[:, h] = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[:, h][:, None])
        out[:, h], spread[:, h] = p @ vv, p @ vv.abs()
    return out, lse, spread, terms


def accept(tokens, target, parent, max_path):
    """(path, the token that follows it) of one sequence."""
    path, n = [], len(tokens)
    at = 0 if n else None
    while at is not None and len(path) < max_path:
        path.append(at)
        at = next((i for i in range(at + 1, n) if (i - 1 if parent is None else parent[i]) == at and tokens[i] == target[at]), None)
    return path, (target[path[-1]] if path else -1)


def random_tree(rng, n, roots=1):
    return [-1 if i < roots else int(rng.integers(0, i)) for i in range(n)]
