"""Paged attention where the values themselves are the difficulty: long flat tails below a peak, V that is not finite; and requests by
themselves, and under tables of the most columns."""
import numpy as np
import pytest
import torch

import paged_ref as R
from paper_2605_25716_amd import binding as fb
from test_gpu_paged import DT, FILL, _attn, _attn_case, i32

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("spread", [0.0, 1.0], ids=["equal", "spread"])
@pytest.mark.parametrize("above,N", [(14.0, 20000), (16.0, 32768), (17.5, 131072)])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("B,n", [(512, 1), (256, 32)], ids=["tokens", "chunks"])
def test_attn_flat_tails(B, n, dt, above, N, spread):
    """A few keys far above tens of thousands of others, which have a good part of the sum only all together: none of it is lost
    in the probabilities' narrowing.  So many requests, all of the same pages, that a workgroup has a long run of them.
    Beside the tolerance of the other tests: fp16's second term ends at steps of 2^-24 and the largest probability is 2^15, so that
    each is off by 2^-25 / 2^15 = 2^-40 at most, relative to 1."""
    page, d = 256, 64
    g = torch.Generator().manual_seed(N)
    K, V = torch.zeros((N, d)), torch.randn((N, d), generator=g)
    K[:, 1] = spread * torch.randn(N, generator=g)
    tops = torch.cat([torch.arange(0, 128, 32), N - 1 - torch.arange(0, 128, 32)])  # before and behind the others, for each wave
    K[tops, 0] = above
    V[:, 0] = 1.0   # an average of ones
    V[:, 2] = 1.0   # the tail by itself
    V[tops, 1:3] = 0.0
    Q = torch.zeros((1, 1, d))
    Q[..., :2] = 8.0  # times 1 / sqrt(64): logits are K's channels 0 and 1
    Q, K, V = (x.to(DT[dt]) for x in (Q, K, V))
    pages = [torch.nn.functional.pad(x, (0, 0, 0, -N % page)).view(-1, 1, page, d).to(DEV) for x in (K, V)]
    T = B * n
    O, lse = fb.fedrag_paged_attn(Q.to(DEV).expand(1, T, d), *pages, torch.arange(pages[0].shape[0], dtype=torch.int32, device=DEV).repeat(B, 1),
                                  i32(np.arange(B + 1) * n), i32([N] * B), n, causal=False)
    k, v, q = K.double().numpy(), V.double().numpy(), Q.double().numpy()[0, 0]
    x = (k @ q) / 8
    p = np.exp(x - x.max())
    total = p.sum()
    off = 16 * R.U / 8 * (np.abs(k) @ np.abs(q)).max() + 8 * R.U * np.sqrt(N)
    tol = (2 * off + 2.0 ** -21 + 2.0 ** -16) * (p @ np.abs(v)) / total + (2.0 ** -40 if dt == "f16" else 0.0) * np.abs(v).sum(0) / total
    want, want_lse = p @ v / total, x.max() + np.log(total)
    worst = (np.abs(O[0, 0].double().cpu().numpy() - want) / tol).max()
    assert worst <= 1, f"{worst:.1f} times the tolerance"
    tol_l = off + 4 * R.U * abs(want_lse) + 2.0 ** -20
    assert np.abs(lse.double().cpu().numpy() - want_lse).max() <= tol_l


ODD = {
    "tokens": ([1, 1, 1], [300, 2500, 33]),
    "few": ([3, 2], [40, 700]),
    "chunks": ([40, 150, 17], [80, 900, 2100]),
    "mixed": ([1, 130, 2], [900, 130, 64]),
}


@pytest.mark.parametrize("scale", [None, 4.0], ids=["", "far"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("dt,d", [("bf16", 128), ("bf16", 64), ("f16", 128), ("f16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("name", list(ODD))
def test_attn_values_that_are_not_finite(name, dt, d, causal, scale):
    """A row that sees a token whose V is not finite has it in those channels: an infinity, or not a number where there are two of
    both signs, whichever tokens other rows see and however small the probability.  (far: logits some hundreds apart, with
    probabilities that are 0 in fp32, and not in 64 bits.)"""
    q, kv = ODD[name]
    Q, Kp, Vp, table, q_start, lens = case = _attn_case(q, kv, 8, 2, d, 16, dt)
    inf = float("inf")
    for b, L in enumerate(kv):
        for t, values in ((L // 9, {3: inf, 4: -inf, 5: inf, 40: inf}), (L * 6 // 10, {5: -inf, 6: float("nan"), 41: -inf}), (L - 1, {7: inf, d - 1: -inf})):
            for c, x in values.items():
                Vp[table[b, t // 16], :, t % 16, c] = x
    O, lse = _attn(case, causal, scale=scale)
    with np.errstate(invalid="ignore"):
        ref = R.attn_ref(*case, causal, d ** -0.5 if scale is None else scale)
    R.check_attn(O, lse, ref, FILL, name)
    assert np.array_equal(np.isnan(O[0].cpu().numpy()), np.isnan(ref[0]))


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_attn_of_a_request_by_itself(dt, causal):
    """What a request comes to does not hang on those beside it, but for roundings."""
    Q, Kp, Vp, table, q_start, lens = case = _attn_case([1, 50, 1, 5], [3000, 600, 20, 1700], 8, 2, 128, 16, dt)
    O, lse = _attn(case, causal)
    for b in range(4):
        rows = slice(int(q_start[b]), int(q_start[b + 1]))
        alone = (Q[:, rows].contiguous(), Kp, Vp, table[b:b + 1], np.array([0, rows.stop - rows.start]), lens[b:b + 1])
        ref = R.attn_ref(*alone, causal, 128 ** -0.5)
        R.check_attn(*_attn(alone, causal), ref, FILL, f"request {b} alone")
        R.check_attn(O[:, :, rows], lse[:, :, rows], ref, FILL, f"request {b} among others")


@pytest.mark.parametrize("dt,q,Hq,Hkv", [("bf16", [1, 1], 600, 300), ("bf16", [20], 256, 128), ("f16", [20, 1, 1], 256, 128), ("f32", [1, 1], 600, 300),
                                         ("f32", [20], 128, 64)])
def test_attn_under_the_widest_table(dt, q, Hq, Hkv):
    """As many columns as a table may have, nearly all of no page.  With so many tiles, the units that the host counts keys in are several
    times their usual length (all units that there might be are below 2^31), and runs and shares are made of those."""
    page, d, kv = 16, 64, [1500, 1111, 33][:len(q)]
    Q, Kp, Vp, table, q_start, lens = _attn_case(q, kv, Hq, Hkv, d, page, dt)
    wide = torch.full((len(q), (2 ** 31 - 256) // page), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = i32(table)
    O, lse = (torch.full((1, Hq, sum(q)) + s, FILL, dtype=torch.float32, device=DEV) for s in ((d,), ()))
    fb.fedrag_paged_attn(Q.to(DEV), Kp.to(DEV), Vp.to(DEV), wide, i32(q_start), i32(lens), max(q), O_part=O, lse=lse)
    R.check_attn(O, lse, R.attn_ref(Q, Kp, Vp, table, q_start, lens, True, d ** -0.5), FILL, "wide")
