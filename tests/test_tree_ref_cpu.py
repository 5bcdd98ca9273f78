"""The plain statements of a drafted step against brute force and closed forms (no GPU)."""
from fractions import Fraction
from itertools import product

import numpy as np
import torch

import tree_ref as TR


def test_masks_are_the_ways_up():
    rng = np.random.default_rng(1)
    sizes = [1, 7, 70, 3]
    up, start = TR.trees(rng, sizes, "forest"), TR.starts([1, 7, 70, 3])
    masks, positions, flags = TR.map_ref(up, start, [5, 9, 70, 2], 2, 83)
    for b, n in enumerate(sizes):
        for i in range(n):
            way, at = set(), i
            while at >= 0:
                way.add(at)
                at = int(up[start[b] + at])
            row = masks[start[b] + i]
            assert {j for j in range(128) if row[j // 64] >> j % 64 & 1} == way
            assert positions[start[b] + i] == [5, 9, 70, 2][b] - n + len(way) - 1
    assert flags == [0] * 4 and masks[81] == [0, 0] and positions[81] == -1


def _law(p, q, children):
    """Distribution of the first token behind the root, exactly: children drawn from q (or given, q None), uniform random numbers."""
    V = len(p)
    law = [Fraction(0)] * V
    for xs in product(range(V), repeat=children):
        weight = Fraction(1)
        for x in xs:
            weight *= q[x]
        r, mass = list(p), Fraction(1)
        for x in xs:
            if weight == 0:
                break
            yes = min(Fraction(1), r[x] / (q[x] * mass)) if mass else Fraction(0)
            law[x] += weight * yes
            weight *= 1 - yes
            r = [max(a - mass * c, 0) for a, c in zip(r, q)]
            mass = sum(r)
        if weight:
            for v in range(V):
                law[v] += weight * (r[v] / mass if mass else p[v])
    return law


def test_the_rule_is_lossless():
    """r <- max(r - M q, 0), accept where u q M < r: the token's law is the target's for any number of siblings."""
    f = lambda *a: [Fraction(x, sum(a)) for x in a]  # noqa: E731
    for p, q in ((f(1, 2, 3), f(3, 1, 1)), (f(5, 1, 1, 1), f(1, 1, 1, 5)), (f(0, 1, 2), f(1, 0, 1)), (f(1, 1), f(1, 1))):
        for children in (1, 2, 3, 4):
            assert _law(p, q, children) == p
    # and taking sum_j M_j q from p at once is the same as taking M q from r each time
    p, q = f(1, 2, 3, 9), f(6, 1, 5, 1)
    r, C, M = list(p), Fraction(0), Fraction(1)
    for _ in range(5):
        r = [max(a - M * c, 0) for a, c in zip(r, q)]
        C += M
        assert r == [max(a - C * c, 0) for a, c in zip(p, q)]
        M = sum(r)


def test_verify_reference_by_hand():
    p = torch.tensor([[0.5, 0.25, 0.25], [0.125, 0.375, 0.5], [1.0, 0.0, 0.0]])
    q = torch.tensor([[0.25, 0.5, 0.25], [0.5, 0.25, 0.25], [0.0, 0.5, 0.5]])
    up, start = [-1, 0, 0], [0, 3]
    run = lambda tokens, u, nxt, most=3, dr=q: [x.tolist() for x in TR.verify_ref(p, dr, tokens, up, start, u, [nxt], most)]  # noqa: E731
    # token 1 drawn at p / q = 1 / 2: accepted below, and then node 1 has no children
    assert run([0, 1, 0], [0, 0.49, 0], 0.6) == [[[0, 1, 0]], [2], [2]]
    # rejected: r = (1/4, 0, 0), M = 1/4; token 0: u q M < r always
    assert run([0, 1, 0], [0, 0.5, 0.99], 0.99) == [[[0, 2, 0]], [2], [0]]
    # both rejected (token 1 twice): C = 5/4, r = (3/16, 0, 0): token 0
    assert run([0, 1, 1], [0, 0.5, 0.0], 0.99) == [[[0, 0, 0]], [1], [0]]
    # no children tried: from p
    assert run([0, 1, 0], [0, 0, 0], 0.5, most=1) == [[[0]], [1], [1]]
    # without distributions of the drafts: token 1 with 1/4, then token 0 with (1/2) / (3/4)
    assert run([0, 1, 0], [0, 0.25, 0.66], 0.0, dr=None) == [[[0, 2, 0]], [2], [0]]
    assert run([0, 1, 0], [0, 0.25, 0.67], 0.0, dr=None) == [[[0, 0, 0]], [1], [2]]


def test_keep_and_trim_references():
    pages = torch.arange(4 * 1 * 16 * 2).view(4, 1, 16, 2).float()
    table = np.array([[2, 0, 1]])
    out = TR.keep_ref(pages, table, [0, 8], [20], np.array([[0, 3, 4, 7]]), [4])
    flat, was = out[[2, 0, 1], 0].view(-1, 2), pages[[2, 0, 1], 0].view(-1, 2)
    assert flat[:20].tolist() == was[[*range(12), 12, 15, 16, 19, 16, 17, 18, 19]].tolist()
    assert torch.equal(out[3], pages[3])
    assert TR.trim_ref([20], [4], table, [7, -1, -1], 1, 16, [0, 8]) == ([16], [7, 0, -1], 2, 0)
    assert TR.trim_ref([20], [0], table, [7, -1], 1, 16) == ([0], [7, 2], 2, 1)
