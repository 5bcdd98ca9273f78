"""Verification by rounds, where the sizes decide how many there are: many requests, with drafts' rows, and vocabularies of up to 256 parts.  Equal
to the plain statement, as everywhere."""
import numpy as np
import pytest

import tree_ref as TR
from test_gpu_tree import _verify, _verify_case


def _case(sizes, V, dt, seed, stubborn, **kw):
    """Stars; the children of `stubborn` requests all have the token of which the draft has most too much: each is rejected, and after each but the
    last a sum over the vocabulary is needed."""
    c = _verify_case(sizes, V, dt, seed, **kw)
    target, draft, tokens, _, start, u, _ = c
    c[3] = TR.trees(np.random.default_rng(1), sizes, "star")
    for b in stubborn:
        root = int(start[b])
        tokens[root:start[b + 1]] = int((draft[root].float() - target[root].float()).argmax())
        u[root:start[b + 1]] = np.nextafter(1.0, 0.0)
    return c


MANY = [3] * 18 + [2, 4, 1, 0] * 4 + [12, 9]  # 36 requests
MANY_CASES = [("f32", 32769), ("f32", 36865), ("bf16", 65551)]
PARTS_CASES = [(dt, V, last) for dt in ("f32", "bf16") for V in (1 << 20, (1 << 20) - 4090) for last in (0, 1)]


def _many(dt, V):
    return _case(MANY, V, dt, V, (0, 3, 5, 19, 34, 35), noise=2.0)


def _parts(dt, V, last):
    c = _case([5, 3, 2], V, dt, last, (0,), noise=3.0, spread=0.5)
    c[6][:] = [[0.3, np.nextafter(1.0, 0.0), 0.999], [np.nextafter(1.0, 0.0), 0.7, 0.0]][last]
    return c


@pytest.mark.parametrize("dt,V", MANY_CASES[:1] + MANY_CASES[2:])
def test_what_the_cases_ask_for(dt, V):
    """Of the many requests some are done with the first launch's sum, some go on to the next sibling, some outlast four rounds more."""
    c = _many(dt, V)
    kept, n_kept, _ = TR.verify_ref(c[0], c[1], *(np.asarray(x) for x in c[2:4]), *c[4:], 5)
    sums = {max(n - 2, 0) if k == 1 else int(path[1]) - 1 for n, k, path in zip(MANY, n_kept, kept) if n}
    assert {0, 1, 2, 7, 10} <= sums


@pytest.mark.gpu
@pytest.mark.parametrize("dt,V", MANY_CASES)
def test_many_requests(dt, V):
    c = _many(dt, V)
    assert _verify(*c, 5)[1][-2:].tolist() == [1, 1]
    c[3] = TR.trees(np.random.default_rng(3), MANY)
    _verify(*c, 5)


@pytest.mark.gpu
@pytest.mark.parametrize("dt,V,last", PARTS_CASES)
def test_as_many_parts_as_there_are(dt, V, last):
    """2^20 tokens and a few less, 256 parts: a thread's sum each.  Three sums of one request, which are more than the two rounds behind the first;
    next tokens in the first part, others and the last."""
    ref = _verify(*_parts(dt, V, last), 3)
    assert ref[1][0] == 1 and (ref[2] // 4096 == 255).any()
