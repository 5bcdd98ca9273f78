"""Paged attention where the values themselves are the difficulty: long flat tails below a peak."""
import numpy as np
import pytest
import torch

import paged_ref as R
from paper_2605_25716_amd import binding as fb
from test_gpu_paged import DT, i32

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("spread", [0.0, 1.0], ids=["equal", "spread"])
@pytest.mark.parametrize("above,N", [(14.0, 20000), (16.0, 32768), (17.5, 131072)])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("B,n", [(512, 1), (256, 32)], ids=["tokens", "chunks"])
def test_attn_flat_tails(B, n, dt, above, N, spread):
    """A few keys far above tens of thousands of others, which have a good part of the sum only all together: none of it is lost
    in the probabilities' narrowing.  So many requests, all of the same pages, that a workgroup has a long run of them.
    Beside the tolerance of the other tests: fp16's second term ends at 2^-24, 2^-40 of the largest probability (2^15), so that
    each is off by half of that at most, relative to 1."""
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
    tol = (2 * off + 2.0 ** -21 + 2.0 ** -16) * (p @ np.abs(v)) / total + (2.0 ** -41 if dt == "f16" else 0.0) * np.abs(v).sum(0) / total
    want, want_lse = p @ v / total, x.max() + np.log(total)
    worst = (np.abs(O[0, 0].double().cpu().numpy() - want) / tol).max()
    assert worst <= 1, f"{worst:.1f} times the tolerance"
    tol_l = off + 4 * R.U * abs(want_lse) + 2.0 ** -20
    assert np.abs(lse.double().cpu().numpy() - want_lse).max() <= tol_l
