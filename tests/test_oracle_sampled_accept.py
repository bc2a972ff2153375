"""Pins of the oracle of acceptance by random numbers: whatever the drafter does, the token that a
node emits first has the target's distribution."""
import itertools

import numpy as np
import pytest

from oracle import sampled_accept as sa


def _first_token_distribution(p, q, kids):
    """Distribution of the token behind a root with these children (accepted child or draw)."""
    out, rest, gone, reach = np.zeros(len(p)), p, 0.0, 1.0
    for x in kids:
        a = sa.acceptance(rest, gone, q, x)
        out[x] += reach * a
        reach *= 1.0 - a
        gone += rest[x]
        rest = sa.refuse(rest, q, x)
    if reach > 0 and rest.sum() > 0:
        out += reach * rest / rest.sum()
    return out


@pytest.mark.parametrize("V,kids,seed", [(2, 1, 0), (3, 2, 1), (4, 3, 2), (5, 2, 3), (3, 4, 4)])
def test_drawn_children_keep_the_targets_distribution(V, kids, seed):
    rng = np.random.default_rng(seed)
    for trial in range(5):
        p, q = rng.dirichlet(np.ones(V) * 0.7), rng.dirichlet(np.ones(V) * 0.7)
        total = np.zeros(V)
        for draft in itertools.product(range(V), repeat=kids):
            total += np.prod(q[list(draft)]) * _first_token_distribution(p, q, draft)
        assert np.allclose(total, p, atol=1e-12)


@pytest.mark.parametrize("V", [2, 3, 5])
def test_chosen_children_keep_the_targets_distribution(V):
    rng = np.random.default_rng(V)
    p = rng.dirichlet(np.ones(V))
    for n in range(V + 1):
        for kids in itertools.permutations(range(V), n):
            assert np.allclose(_first_token_distribution(p, None, kids), p, atol=1e-12)
    assert np.allclose(_first_token_distribution(p, None, (1, 1, 0)), p, atol=1e-12)      # a token twice


@pytest.mark.parametrize("drawn", [True, False])
def test_the_walk_follows_the_acceptance_probabilities(drawn):
    """Random numbers just below and just above the thresholds decide as `acceptance` says."""
    rng = np.random.default_rng(11)
    parent, V = [-1, 0, 0, 1, 1, 2], 6
    for trial in range(200):
        p, q = rng.dirichlet(np.ones(V), size=6), rng.dirichlet(np.ones(V), size=6) if drawn else None
        tok, u = rng.integers(0, V, 6), rng.random(6)
        r = sa.sampled_accept(parent, tok + 10, p, q, 10, u, rng.random(), 7)
        assert r["length"] == len(r["path"]) - 1 and r["best"] == r["path"][-1] and len(r["tokens"]) == r["length"] + 1
        for up, down in zip(r["path"], r["path"][1:]):
            assert parent[down] == up
        kids = [c for c in range(6) if parent[c] == 0]
        rest, gone = p[0], 0.0
        for c in kids:
            a = sa.acceptance(rest, gone, q[0] if drawn else None, tok[c])
            if u[c] < a:
                assert r["path"][1] == c
                break
            gone += rest[tok[c]]
            rest = sa.refuse(rest, q[0] if drawn else None, tok[c])
        else:
            assert r["length"] == 0


def test_equal_distributions_accept_everything_and_depth_is_capped():
    p = np.full((4, 4), 0.25)
    for cap in (0, 1, 2, 3, 7):
        r = sa.sampled_accept([-1, 0, 1, 2], [0, 1, 2, 3], p, p, 0, [0.999] * 4, 0.5, cap)
        assert r["length"] == min(3, cap) and r["tokens"][-1] == 2


def test_draw_edges():
    p = np.array([0.0, 0.5, 0.0, 0.5, 0.0])
    assert sa.draw(p, p, 0.0) == (1, 0) and sa.draw(p, p, 0.5) == (3, 0) and sa.draw(p, p, 1.0) == (3, 0)
    assert sa.draw(np.zeros(5), p, 0.0) == (1, 1) and sa.draw(np.zeros(5), np.zeros(5), 0.3) == (0, 3)
