"""Attention by masks in 16 bits: how many bits a probability has in the second product.

With u = 2^-24.  The scores here are exact: one channel of Q and K is not zero, and a product of two 16-bit values fits fp32.

A token alone.  Its probability is a power of two, exactly: the exponent's argument is the difference of two equal roundings.  V times it, the sum
and the other waves' (0) are exact too; the division, and the fold of a cut row, round: 2^-23 of |V|.
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
