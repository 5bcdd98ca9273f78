"""Attention by masks in 16 bits: how many bits a probability has in the second product.

With u = 2^-24.  The scores here are exact: one channel of Q and K is not zero, and a product of two 16-bit values fits fp32.

A token alone.  Its probability is a power of two, exactly: the exponent's argument is the difference of two equal roundings.  V times it, the sum
and the other waves' (0) are exact too; the division, and the fold of a cut row, round: 2^-23 of |V|.

Few tokens.  |scale s log2 e| <= X = 1.36 for all of a row's tokens, of which three at most have a probability that is not 0.
  exponent    log2 e and its product with the scale are rounded, then the product with s, that of the maximum alike, and the difference (below 2 X):
              (2 + 1 + 2 + 1 + 2) u X < 11 u; fp16: the reference, 15 below the maximum, is rounded to 2^-21 at most (8 u, the same for a row's
              tokens), and so the difference, of up to 16 to 2^-21: 8 u more for each.  Times ln 2: 8 u, or 14 u.
  2^x         a step: 2 u.
              Both for the probability and for the sum that it is divided by: 20 u, or 32 u.
  sums        of three terms, in the numerator by up to three products each, in any order, and the rest 0: 9 u and 3 u; the waves' fold and the
              quotient: 4 u.
  terms       bf16: of 24 significant bits the first term leaves 16 at most, the second 8, and the third takes them: 0.  Two terms: 2^-8 of what the
              first leaves, 2^-8 of the value: 2^-16.  fp16: 2^-11 twice, 2^-22.
All are relative to sum p |v|: 36 u (48 u in fp16) and the terms.
"""
import numpy as np
import pytest
import torch

from paper_2605_25716_amd import binding as fb

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24


def _run(q, k, V, G, sees, before, dt, scale, page=16):
    """Rows' and tokens' values in channel 0 (q [T, G], k [kv]) and V [kv, d]; sees: bool [T, T], of the last T tokens.  One KV head twice, as two."""
    T, kv, d = q.shape[0], len(k), V.shape[1]
    assert kv == before + T
    pages = -(-kv // page)
    Kp, Vp = (torch.zeros((pages, 2, page, d), dtype=DT[dt]) for _ in range(2))
    token = torch.arange(kv)
    Kp[token // page, :, token % page, 0] = torch.tensor(k).to(DT[dt])[:, None]
    Vp[token // page, :, token % page] = V[:, None]
    Q = torch.zeros((2 * G, T, d), dtype=DT[dt])
    Q[:, :, 0] = torch.tensor(q).T.repeat(2, 1).to(DT[dt])
    words = -(-T // 64)
    mask = np.zeros((T, words), np.uint64)
    for t in range(T):
        for j in np.nonzero(sees[t])[0]:
            mask[t, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    O, lse = fb.fedrag_paged_tree_attn(Q.to(DEV), Kp.to(DEV), Vp.to(DEV), i32([list(range(pages))]), i32([0, T]), i32([kv]),
                                       torch.from_numpy(mask.view(np.int64)).to(DEV), T, softmax_scale=scale)
    return O[0].double().cpu().numpy().reshape(2, G, T, d), lse[0].double().cpu().numpy().reshape(2, G, T)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 16), (3, 4), (4, 8), (7, 4), (8, 4), (9, 4), (16, 4), (33, 1), (8, 8)])
def test_a_token_alone(dt, T, G):
    """Rows that see one token, at scores of either sign of up to 3 * 10^5, in requests of 1 to 64 rows a KV head: its V."""
    rng = np.random.default_rng(T * G)
    as_stored = lambda x: torch.tensor(x).to(DT[dt]).double().numpy()  # noqa: E731
    for sees in (np.eye(T, dtype=bool), np.eye(T, dtype=bool)[rng.integers(0, T, T)]):
        q, k = as_stored(rng.uniform(-900, 900, (T, G))), as_stored(rng.uniform(1, 1000, T))
        V = torch.tensor(rng.standard_normal((T, 128))).to(DT[dt])
        O, lse = _run(q, k, V, G, sees, 0, dt, 0.34)
        at = sees.argmax(1)
        v, score = V.double().numpy()[at], (q * k[at][:, None]).T * float(np.float32(0.34))
        assert (np.abs(O - v) <= 2 * U * np.abs(v)).all(), np.max(np.abs(O - v) / np.abs(v)) / U
        assert (np.abs(lse - score) <= 8 * U * np.abs(score) + 2.0 ** -20).all()


def _few(dt, T, G, before, seed):
    """Rows that see three tokens: two of their own by the mask, and one of before where there are such (all the others there far below)."""
    rng = np.random.default_rng(seed)
    as_stored = lambda x: torch.tensor(x).to(DT[dt]).double().numpy()  # noqa: E731
    q, k = as_stored(rng.uniform(0.5, 1.25, (T, G))), as_stored(rng.uniform(-1.5, 1.5, before + T))
    if before:
        keep = int(rng.integers(0, before))
        k[:before][np.arange(before) != keep] = -4096.0
    V = torch.tensor(rng.standard_normal((before + T, 128))).to(DT[dt])
    sees = np.eye(T, dtype=bool)
    sees[np.arange(T), rng.integers(0, T, T)] = True
    return q, k, V, sees


def _few_ref(q, k, V, sees, before, scale, terms=None):
    """(O [G, T, d], its sum p |v|); terms: probabilities relative to the largest in so many bf16 terms in the product alone"""
    T, G = q.shape
    O, size = np.zeros((G, T, 128)), np.zeros((G, T, 128))
    v = V.double().numpy()
    for t in range(T):
        there = np.concatenate([np.ones(before, bool), sees[t]])
        x = scale * q[t][:, None] * k[there]
        p = np.exp(x - x.max(1, keepdims=True))
        used = p
        if terms:
            rest, used = torch.tensor(p).float(), torch.zeros(p.shape, dtype=torch.float64)
            for _ in range(terms):
                term = rest.bfloat16().float()
                used, rest = used + term.double(), rest - term
            used = used.numpy()
        O[:, t], size[:, t] = used @ v[there] / p.sum(1, keepdims=True), p @ np.abs(v[there]) / p.sum(1, keepdims=True)
    return O, size


FEW = [(1, 8, 40), (4, 4, 0), (4, 4, 200), (6, 5, 0), (8, 4, 70), (32, 1, 600), (16, 4, 0), (60, 1, 130), (70, 4, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,G,before", FEW)
def test_terms_of_a_probability(dt, T, G, before):
    scale, rows = 0.5, T * G
    for seed in range(6):
        case = _few(dt, T, G, before, seed)
        O, _ = _run(*case[:3], G, case[3], before, dt, scale)
        ref, size = _few_ref(*case, before, scale)
        terms = 2.0 ** -22 if dt == "f16" else 0.0 if rows <= 32 else 2.0 ** -16
        off = np.abs(O - ref) / size
        print(f"{dt} {T} {G} {before} {seed}: {off.max() / U:.1f} u", flush=True)
        assert (off <= (36 if dt == "bf16" else 48) * U + terms).all(), off.max() / U


def test_a_term_less_would_show():
    """The same inputs with a term less, in the reference: more than twice the bound off, where three terms are exact."""
    for T, G, before in FEW:
        if T * G > 32 or T == 1:
            continue
        worst = 0.0
        for seed in range(6):
            case = _few("bf16", T, G, before, seed)
            ref, size = _few_ref(*case, before, 0.5)
            worst = max(worst, (np.abs(_few_ref(*case, before, 0.5, terms=2)[0] - ref) / size).max())
            assert (np.abs(_few_ref(*case, before, 0.5, terms=3)[0] - ref) <= U * size).all()
        print(f"{T} {G} {before}: {worst / U:.1f} u", flush=True)
        assert worst > 2 * 36 * U
