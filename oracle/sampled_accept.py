"""CPU oracle for acceptance by random numbers.  TEST INFRASTRUCTURE ONLY (same rules as
verify_oracle.py: tests may import it; the product never does).

The paper accepts by bins of the greedy token (Sec. 4.3).  This is the other rule of speculative
decoding, the one that keeps the target's distribution (accept a drawn token x with probability
min(1, p(x) / q(x)), otherwise go on with the normalised positive part of p - q), carried over to a
tree: the children of a node are tried in ascending order, each against what the refusals before it
have left.  Children that were chosen instead of drawn (no q) are accepted with their share of what
is left, and are taken out of it when refused.

The residual distribution itself is carried along here, normalised after every refusal; the product
carries two numbers in its place.  Pinned in tests/test_oracle_sampled_accept.py: the emitted token
has the target's distribution, by summing over every draft and integrating the random numbers out.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence

import numpy as np


def refuse(rest: np.ndarray, q: Optional[np.ndarray], x: int) -> np.ndarray:
    """What is left of a node's distribution when its child with token column x was refused.  Not
    drawn (q None): unnormalised, with x gone."""
    if q is None:
        out = rest.copy()
        if 0 <= x < len(rest):
            out[x] = 0.0
        return out
    out = rest - q
    out = np.where(out > 0, out, 0.0)
    return out / out.sum() if out.sum() > 0 else out


def acceptance(rest: np.ndarray, gone: float, q: Optional[np.ndarray], x: int) -> float:
    """Probability that the child with token column x is accepted; gone: mass of earlier refusals."""
    px = rest[x] if 0 <= x < len(rest) else 0.0
    if not px > 0:
        return 0.0
    share = q[x] if q is not None else max(1.0 - gone, 0.0)
    return 1.0 if share <= px else px / share


def draw(rest: np.ndarray, p: np.ndarray, u: float):
    """(column, status): the first column at which the cumulated sum exceeds u * total."""
    status = 0
    if not rest.sum() > 0:
        status, rest = 1, p
        if not rest.sum() > 0:
            return 0, 3
    cum = np.cumsum(rest)
    above = np.flatnonzero((cum > u * cum[-1]) & (rest > 0))
    return int(above[0] if len(above) else np.flatnonzero(rest > 0)[-1]), status


def sampled_accept(parent: Sequence[int], draft_token: Sequence[int], target_prob: np.ndarray,
                   draft_prob: Optional[np.ndarray], lo: int, u_accept: Sequence[float], u_draw: float,
                   d_cap: int) -> Dict:
    """target_prob, draft_prob: float64 [T, V].  Returns dict: mask, length, best, path, tokens, status."""
    clean = lambda r: np.where(np.isnan(r) | (r < 0), 0.0, r)
    T, node, path, tokens = len(parent), 0, [0], []
    while True:
        p = clean(target_prob[node])
        q = clean(draft_prob[node]) if draft_prob is not None else None
        rest, gone, down = p, 0.0, None
        kids: List[int] = [c for c in range(node + 1, T) if parent[c] == node] if len(path) <= d_cap else []
        for c in kids:
            x = int(draft_token[c]) - lo
            px = rest[x] if 0 <= x < len(rest) else 0.0
            share = (q[x] if 0 <= x < len(rest) else 0.0) if q is not None else max(1.0 - gone, 0.0)
            if px > 0 and u_accept[c] * share < px:
                down = c
                break
            gone += px
            rest = refuse(rest, q, x)
        if down is None:
            break
        tokens.append(int(draft_token[down]))
        path.append(down)
        node = down
    col, status = draw(rest, p, u_draw)
    mask = np.zeros(T, dtype=bool)
    mask[path] = True
    return {"mask": mask, "length": len(path) - 1, "best": node, "path": path, "tokens": tokens + [lo + col],
            "status": status}
