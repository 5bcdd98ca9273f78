"""A drafted step's calls on the GPU: masks, attention, verification, the rows that stay and the pages that go, each against its plain
statement."""
import numpy as np
import pytest
import torch

import paged_ref as R
import tree_ref as TR
from paper_2605_25716_amd import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FILL = 7.0


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int64).astype(np.int32)).to(DEV)


# ----------------------------------------------------------------------------------------------- masks
def _map(parents, q_start, kv, words, T):
    mask = torch.full((T, words), 5, dtype=torch.int64, device=DEV)
    positions, flags = (torch.full((n,), 5, dtype=torch.int32, device=DEV) for n in (T, len(kv)))
    up = np.concatenate([parents, np.full(T, 3)])[:T]
    fb.fedrag_tree_map(i32(up), i32(q_start), i32(kv), words, tree_mask=mask, positions=positions, flags=flags)
    ref = TR.map_ref(up, q_start, kv, words, T)
    np.testing.assert_array_equal(mask.cpu().numpy(), TR.signed(ref[0]).reshape(T, words))
    assert positions.tolist() == ref[1] and flags.tolist() == ref[2]
    return mask


@pytest.mark.parametrize("shape", ["tree", "chain", "star", "forest"])
@pytest.mark.parametrize("sizes,words,pad", [([1], 1, 0), ([5], 1, 3), ([64], 1, 0), ([65, 1, 63], 2, 5), ([0, 7, 0], 1, 70), ([300, 2, 128, 129], 5, 1),
                                             ([4096], 64, 2), ([3] * 257, 3, 300)])
def test_masks(shape, sizes, words, pad):
    rng = np.random.default_rng(len(sizes) + words)
    up = TR.trees(rng, sizes, shape)
    _map(up, TR.starts(sizes), [n + int(rng.integers(0, 50)) for n in sizes], words, sum(sizes) + pad)


@pytest.mark.parametrize("what", ["parents", "words", "short_kv", "beyond_rows", "no_requests", "negative_kv"])
def test_masks_out_of_the_ordinary(what):
    rng = np.random.default_rng(7)
    sizes, words, T = [70, 200, 3], 4, 280
    up, start, kv = TR.trees(rng, sizes, "forest"), TR.starts(sizes), [90, 300, 3]
    if what == "parents":
        up[[3, 75, 150, 269, 272]] = [3, 2000, -2 ** 31, 2 ** 31 - 1, -2]
    if what == "words":
        words = 1
        up[70:270] = np.maximum(up[70:270], np.arange(-1, 199) - 3)
    if what == "short_kv":
        kv = [10, 200, 0]
    if what == "beyond_rows":
        T = 100
    if what == "negative_kv":
        kv = [-5, 200, 3]
    if what == "no_requests":
        start, kv, up = [0], [], np.zeros(0, np.int64)
    _map(up, start, kv, words, T)


def test_masks_without_positions_kept_apart():
    up, start = TR.trees(np.random.default_rng(2), [20, 9]), TR.starts([20, 9])
    a = fb.fedrag_tree_map(i32(up), i32(start), i32([30, 9]), 1)
    assert TR.signed(TR.map_ref(up, start, [30, 9], 1, 29)[0]).tolist() == a[0].tolist()


# ----------------------------------------------------------------------------------------------- attention
def _attn_case(sizes, kv, Hq, Hkv, d, page, dt, seed, pad=0, words=None, shape="tree", mask=None, columns_more=1, big=0.0):
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    T = sum(sizes) + pad
    need = [-(-n // page) for n in kv]
    n_pages = sum(need) + 3
    ids = rng.permutation(n_pages)
    table = np.full((len(kv), max(need) + columns_more), -1)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    Kp, Vp = (torch.randn((n_pages, Hkv, page, d), generator=g).to(DT[dt]) for _ in range(2))
    if big:
        Kp *= big
    Q = torch.randn((T, Hq, d), generator=g).to(DT[dt]).transpose(0, 1)
    start = TR.starts(sizes)
    words = words or max(1, -(-max(sizes) // 64))
    if mask is None:
        mask = np.zeros((T, words), np.int64)
        ref = TR.map_ref(TR.trees(rng, sizes, shape), start, kv, words, T)[0]
        mask = TR.signed(ref).reshape(T, words)
    elif mask == "random":
        mask = rng.integers(-2 ** 63, 2 ** 63 - 1, (T, words))
    elif mask == "none":
        mask = np.zeros((T, words), np.int64)
    return dict(Q=Q, Kp=Kp, Vp=Vp, table=table, start=start, kv=kv, mask=mask, max_q=max(sizes), d=d)


def _attn(c, max_q=None, check=True, what="", **kw):
    Hq, T, d = c["Q"].shape
    O = torch.full((1, Hq, T, d), FILL, device=DEV)
    lse = torch.full((1, Hq, T), FILL, device=DEV)
    Q = c["Q"].transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
    fb.fedrag_paged_tree_attn(Q, c["Kp"].to(DEV), c["Vp"].to(DEV), i32(c["table"]), i32(c["start"]), i32(c["kv"]),
                              torch.from_numpy(np.ascontiguousarray(c["mask"])).to(DEV), c["max_q"] if max_q is None else max_q, O_part=O, lse=lse, **kw)
    if check:
        R.check_attn(O, lse, TR.attn_ref(c["Q"], c["Kp"], c["Vp"], c["table"], c["start"], c["kv"], c["mask"], d ** -0.5), FILL, what)
    return O, lse


SIZES = [([1], [1]), ([1], [193]), ([4], [200]), ([3], [3]), ([16], [700]), ([33], [40]), ([65], [300]), ([7, 1, 0, 20], [50, 900, 30, 20]),
         ([64, 130, 2], [64, 150, 1100]), ([300], [400])]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("Hq,Hkv,d,page", [(8, 2, 128, 16), (7, 1, 64, 64), (4, 4, 128, 256), (32, 2, 64, 32)])
def test_attention(dt, Hq, Hkv, d, page):
    for k, (sizes, kv) in enumerate(SIZES):
        case = _attn_case(sizes, kv, Hq, Hkv, d, page, dt, seed=k, pad=k % 3)
        for max_q in {max(sizes), 0} | ({1} if k % 2 else set()):  # (which kernels run, never the result)
            _attn(case, max_q, what=f"{sizes} {kv} {max_q}")


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("mask", ["random", "none"])
def test_any_bits(dt, mask):
    """Bits of nodes that are no ancestors, of later ones and of none; rows without any, also where there is nothing before them."""
    for k, (sizes, kv) in enumerate([([5, 70, 1], [5, 100, 1]), ([3], [3]), ([40, 9], [333, 9]), ([130], [130])]):
        for words in (1, 3):
            _attn(_attn_case(sizes, kv, 8, 2, 128, 16, dt, seed=k, mask=mask, words=words), what=f"{sizes} {words}")
            _attn(_attn_case(sizes, kv, 5, 1, 64, 128, dt, seed=k, mask=mask, words=words), what=f"{sizes} {words}")


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_tail_at_every_place_of_a_tile(dt):
    """Trees that begin and end anywhere in a tile of keys and in a word of the mask."""
    for n in (2, 20, 65):
        sizes = [n] * 9
        kv = [n + 120 + 7 * i for i in range(8)] + [n + 64]
        _attn(_attn_case(sizes, kv, 4, 1, 128, 16, dt, seed=n, mask="random"), what=f"{n}")


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [3, 30, 100])
def test_a_chain_is_causal(dt, n):
    c = _attn_case([n, n], [700, n], 8, 2, 128, 32, dt, seed=n, shape="chain")
    O, lse = _attn(c)
    ref = fb.fedrag_paged_attn(c["Q"].to(DEV), c["Kp"].to(DEV), c["Vp"].to(DEV), i32(c["table"]), i32(c["start"]), i32(c["kv"]), n, causal=True)
    _, _, t_o, t_l, _ = TR.attn_ref(c["Q"], c["Kp"], c["Vp"], c["table"], c["start"], c["kv"], c["mask"], 128 ** -0.5)
    assert ((O - ref[0])[0].abs().double().cpu().numpy() <= 2 * t_o).all() and ((lse - ref[1])[0].abs().double().cpu().numpy() <= 2 * t_l).all()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes,kv", [([4], [100]), ([40], [70]), ([100], [200])])
def test_what_a_row_does_not_see_does_not_touch_it(dt, sizes, kv):
    """NaN and infinities in K and V of nodes that are not ancestors, of missing pages and behind the request."""
    for bad in (float("nan"), float("inf"), -float("inf")):
        c = _attn_case(sizes, kv, 8, 2, 128, 16, dt, seed=3, shape="star")
        n, L = sizes[0], kv[0]
        clean = TR.attn_ref(c["Q"], c["Kp"], c["Vp"], c["table"], c["start"], c["kv"], c["mask"], 128 ** -0.5)
        for node in range(1, n, 2):  # (siblings: only their own rows see them)
            t = L - n + node
            c["Kp"][c["table"][0, t // 16], :, t % 16] = bad
            c["Vp"][c["table"][0, t // 16], :, t % 16, node % 128] = bad
        if L % 16:
            c["Kp"][c["table"][0, L // 16], :, L % 16:] = bad
            c["Vp"][c["table"][0, L // 16], :, L % 16:] = bad
        O, lse = _attn(c, check=False)
        rows = np.arange(0, n, 2)
        got, want, tol = O[0].double().cpu().numpy()[:, rows], clean[0][:, rows], clean[2][:, rows]
        assert (np.abs(got - want) <= tol).all(), bad
        assert (np.abs(lse[0].double().cpu().numpy()[:, rows] - clean[1][:, rows]) <= clean[3][:, rows]).all()
        assert not np.isfinite(O[0].cpu().numpy()[:, 1::2]).all(axis=-1).any()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [3, 40, 140])
def test_values_that_are_not_finite_where_they_are_seen(dt, n):
    """V alone: that channel of the rows that see it, an infinity or not a number, and nothing else."""
    c = _attn_case([n], [n + 90], 8, 2, 128, 16, dt, seed=5)
    rng = np.random.default_rng(1)
    for k in range(6):
        t = int(rng.integers(80, n + 90))
        c["Vp"][c["table"][0, t // 16], :, t % 16, 10 * k] = [float("inf"), -float("inf"), float("nan")][k % 3]
    t = n + 89
    c["Vp"][c["table"][0, t // 16], 1, t % 16, 100] = float("inf")
    with np.errstate(invalid="ignore"):
        _attn(c)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_missing_pages_and_columns(dt):
    for hole in (-1, 10 ** 6):
        c = _attn_case([40, 6, 90], [200, 77, 333], 8, 2, 128, 16, dt, seed=9)
        c["table"][0, 3], c["table"][0, 11], c["table"][2, 20], c["table"][1, :] = hole, hole, hole, hole
        _attn(c)
    c = _attn_case([40, 6, 90], [200, 77, 333], 8, 2, 128, 16, dt, seed=9)
    c["table"] = c["table"][:, :9]  # too few columns: the trees of two requests lie behind them, and part of the tokens before
    _attn(c)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rows_and_lengths_at_odds(dt):
    """More rows than tokens; starts outside the rows; lengths below zero."""
    c = _attn_case([20, 9, 30], [64, 40, 64], 8, 2, 64, 16, dt, seed=4, mask="random")
    _attn({**c, "kv": [12, 40, 3]}, what="rows without tokens")
    _attn({**c, "kv": [64, -3, 0]}, what="no tokens")
    _attn({**c, "start": np.array([-4, 20, 29, 90])}, what="starts")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_long_requests_cut_into_runs(dt):
    """Keys of one request over many workgroups, whose partials are folded, the tree in the last of them or across two."""
    for sizes, kv in (([6], [20000]), ([40], [9000]), ([70, 1, 13], [5000, 7000, 4100])):
        Hq = 8
        _attn(_attn_case(sizes, kv, Hq, 2, 128, 64, dt, seed=1), what=f"{sizes}")


def test_large_scores_stay_apart():
    """Scores of some hundred: a row's probabilities sit on few tokens, nodes among them."""
    for dt in ("f32", "bf16", "f16"):
        for n in (5, 40):
            _attn(_attn_case([n], [n + 100], 8, 2, 128, 16, dt, seed=n, big=6.0), what=dt)


# ----------------------------------------------------------------------------------------------- verification
def _verify(target, draft, tokens, up, start, u, u_next, most, **kw):
    B = len(start) - 1
    kept = torch.full((B, most), 9, dtype=torch.int32, device=DEV)
    n_kept, nxt = (torch.full((B,), 9, dtype=torch.int32, device=DEV) for _ in range(2))
    f64 = lambda x: torch.as_tensor(np.asarray(x, dtype=np.float64)).to(DEV)  # noqa: E731
    on = lambda x: None if x is None else x if x.is_cuda else x.to(DEV)  # noqa: E731
    fb.fedrag_tree_verify(on(target), i32(tokens), i32(up), i32(start), f64(u), f64(u_next), draft=on(draft), kept=kept, n_kept=n_kept,
                          next_token=nxt, **kw)
    ref = TR.verify_ref(target.cpu(), None if draft is None else draft.cpu(), np.asarray(tokens), np.asarray(up), start, u, u_next, most)
    assert n_kept.tolist() == ref[1].tolist()
    assert kept.tolist() == ref[0].tolist()
    assert nxt.tolist() == ref[2].tolist()
    return ref


def _verify_case(sizes, V, dt, seed, noise=1.0, spread=2.0, with_draft=True):
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    T, start = sum(sizes), TR.starts(sizes)
    up = TR.trees(rng, sizes)
    logits = spread * torch.randn((T, V), generator=g)
    target = torch.softmax(logits, -1).to(DT[dt])
    draft = torch.softmax(logits + noise * torch.randn((T, V), generator=g), -1).to(DT[dt])
    above = np.concatenate([start[b] + np.maximum(up[start[b]:start[b + 1]], 0) for b in range(len(sizes))]).astype(np.int64)
    tokens = torch.multinomial(draft.float()[above], 1, generator=g)[:, 0].numpy() if T else np.zeros(0)
    return [target, draft if with_draft else None, tokens, up, start, rng.random(T), rng.random(len(sizes))]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("V", [1, 2, 9, 255, 4095, 4096, 4097, 8192, 10001])
def test_verify(dt, with_draft, V):
    for sizes, most in (([1], 1), ([6, 1, 0, 12], 12), ([20] * 9, 5), ([70, 3, 150], 40)):
        _verify(*_verify_case(sizes, V, dt, V + len(sizes), with_draft=with_draft), most)


@pytest.mark.parametrize("with_draft", [True, False])
def test_verify_many_siblings_rejected(with_draft):
    """Random numbers near one: one child after the other is rejected, many more than there are rounds; the sums go on and on."""
    for V in (40, 5000, 33000):
        c = _verify_case([30, 80, 9, 2], V, "f32", 3, noise=3.0, with_draft=with_draft)
        c[3] = TR.trees(np.random.default_rng(1), [30, 80, 9, 2], "star")
        c[5] = 1.0 - 1e-9 * np.random.default_rng(2).random(121)
        n = _verify(*c, 8)[1]
        c[5][:] = np.nextafter(1.0, 0.0)
        _verify(*c, 8)
        c[2][:] = c[2][1]  # one token again and again
        _verify(*c, 8)
        assert n.min() >= 1


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_verify_a_vocabulary_of_many_parts(dt):
    for with_draft in (True, False):
        _verify(*_verify_case([9, 5, 17], 50021, dt, 11, with_draft=with_draft), 6)
        for sizes, most in (([1], 1), ([6, 1, 0, 12], 12), ([70, 3, 100], 40)):
            _verify(*_verify_case(sizes, 70001, dt, len(sizes), with_draft=with_draft), most)


@pytest.mark.parametrize("dt, V", [("f32", 32768), ("f32", 32769), ("f32", 32765), ("f32", 3), ("f32", 4), ("f32", 5), ("f32", 28673), ("bf16", 65536),
                                   ("bf16", 65537), ("bf16", 65529), ("f16", 7), ("f16", 8), ("f16", 11), ("f16", 57351)])
def test_verify_where_the_forms_meet(dt, V):
    """Rows that fill one workgroup's registers, or one of its steps, by a token more or less; fewer tokens than a load has."""
    for with_draft in (True, False):
        c = _verify_case([12, 0, 7, 25, 1, 1, 1, 1], V, dt, V, with_draft=with_draft, spread=0.1)
        c[6][:] = [0.0, 0.1, np.nextafter(1.0, 0.0), 0.5, 0.9, 0.99, 0.999, 0.99999]
        _verify(*c, 9)


@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("what", ["extremes", "outside", "nan_u"])
def test_verify_random_numbers_at_their_ends(with_draft, what):
    for V in (3, 4500, 33333):
        c = _verify_case([8] * 6, V, "f32", 5, with_draft=with_draft)
        ends = {"extremes": [0.0, np.nextafter(1.0, 0.0)], "outside": [-1.0, 1.0, 7.0, -np.inf, np.inf], "nan_u": [np.nan, 0.5]}[what]
        rng = np.random.default_rng(2)
        c[5], c[6] = rng.choice(ends, 48), rng.choice(ends, 6)
        _verify(*c, 8)


@pytest.mark.parametrize("dt", ["f32", "f16"])
def test_verify_values_at_their_ends(dt):
    """Rows of zeros, of one token, equal rows, values that are no probabilities; tokens and parents that are none."""
    for V, with_draft in ((4300, True), (4300, False), (70003, True), (70003, False)):
        c = _verify_case([10] * 12, V, dt, 8, with_draft=with_draft)
        t, q = c[0], c[1]
        t[0:10] = 0
        t[10:20] = 0
        t[10:20, V - 1] = 1
        t[20:30] = 1.0
        t[30:40, ::3] = float("nan")
        t[40:50, 7] = float("inf")
        t[50:60, 5] = -1.0
        t[60:70] *= 3.0
        if q is not None:
            q[70:80] = t[70:80]
            q[80:90] = 0
            q[90:100, ::5] = float("nan")
            q[100:110, 3] = float("inf")
            q[20:30] = 1.0
        c[2][[3, 13, 44, 71, 85]] = [-1, V, 2 ** 31 - 1, -2 ** 31, V + 5]
        c[3][[5, 17, 33, 102]] = [5, 900, -7, 9]
        _verify(*c, 10)


def test_verify_rows_with_strides():
    for dt in ("f32", "bf16"):
        for shift in (0, 1, 3):
            for V in (9001, 70001):
                target, draft, *c = _verify_case([6, 9, 4], V, dt, 4)
                wide = torch.zeros((19, V + 99), dtype=DT[dt], device=DEV)
                wide[:, shift:shift + V] = target.to(DEV)
                far = torch.zeros((19, V + 16), dtype=DT[dt], device=DEV)
                far[:, :V] = draft.to(DEV)
                _verify(wide[:, shift:shift + V], far[:, :V], *c, 9)


def test_verify_offsets_beyond_32_bits():
    """Rows whose elements are numbered beyond 2^32."""
    V, rows = 1 << 20, 4200
    target = torch.zeros((rows, V), dtype=torch.bfloat16, device=DEV)  # 8.8 GB
    start = [0, rows - 5, rows]
    g = np.random.default_rng(1)
    for r in (0, *range(rows - 5, rows)):
        target[r, torch.as_tensor(g.choice(V, 3, replace=False)).to(DEV)] = torch.tensor([0.5, 0.25, 0.25], dtype=torch.bfloat16, device=DEV)
    up = np.full(rows, -1)
    up[-4:] = [0, 1, 2, 3]
    tokens = np.zeros(rows, np.int64)
    for i in range(4):
        tokens[rows - 4 + i] = int(target[rows - 5 + i].argmax())
    kept, n_kept, nxt = fb.fedrag_tree_verify(target, i32(tokens), i32(up), i32(start), torch.full((rows,), 0.3, dtype=torch.float64, device=DEV),
                                              torch.tensor([0.99, 0.99], dtype=torch.float64, device=DEV), max_kept=6)
    assert n_kept.tolist() == [1, 5] and kept.tolist() == [[0] * 6, [0, 1, 2, 3, 4, 0]]
    for b, row in enumerate((0, rows - 1)):
        assert int(nxt[b]) == int(target[row].nonzero().max())


def test_verified_tokens_follow_the_target():
    """The law itself: the first token behind the root over 60000 requests of one root, drafts drawn anew for each, against the target's
    probabilities, within five standard deviations (the random numbers are fixed: it passes or it does not)."""
    B, n, V = 60000, 4, 7
    g = torch.Generator().manual_seed(0)
    p, q = torch.softmax(1.5 * torch.randn(V, generator=g), 0), torch.softmax(1.5 * torch.randn(V, generator=g), 0)
    tokens = torch.multinomial(q.repeat(B, 1), n, replacement=True, generator=g)  # four nodes, the first of which is the root
    up = torch.tensor([-1, 0, 0, 0]).repeat(B)
    rand = lambda k: torch.rand(k, generator=g, dtype=torch.float64).to(DEV)  # noqa: E731
    kept, n_kept, nxt = fb.fedrag_tree_verify(p.repeat(B * n, 1).to(DEV), i32(tokens.view(-1)), i32(up), i32(np.arange(0, B * n + 1, n)), rand(B * n),
                                              rand(B), draft=q.repeat(B * n, 1).to(DEV), max_kept=2)
    first = torch.where(n_kept == 2, tokens.to(DEV).int().gather(1, kept[:, 1:].long())[:, 0], nxt)
    share = torch.bincount(first.long().cpu(), minlength=V).double() / B
    assert ((share - p.double()).abs() <= 5 * (p.double() * (1 - p.double()) / B).sqrt()).all(), (share, p)
    assert 0.3 < (n_kept == 2).double().mean() < 1


# ----------------------------------------------------------------------------------------------- what stays
def _bits(x):
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


def _keep_case(sizes, kv, page, seed, most=None):
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in kv]
    ids = rng.permutation(sum(need) + 4)
    table = np.full((len(kv), max(need) + 1), -1)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    n_kept = [int(rng.integers(0, n + 1)) if n else 0 for n in sizes]
    kept = np.zeros((len(kv), most or max(1, max(n_kept))), np.int64)
    for b, (n, k) in enumerate(zip(sizes, n_kept)):
        k = n_kept[b] = min(k, kept.shape[1])
        kept[b, :k] = np.sort(rng.choice(n, k, replace=False))
    return table, TR.starts(sizes), kv, kept, n_kept, sum(need) + 4


def _keep(pools, table, start, kv, kept, n_kept):
    caches = [tuple(x.to(DEV) for x in pool) for pool in pools]
    fb.fedrag_paged_keep(caches, i32(table), i32(start), i32(kv), i32(kept), i32(n_kept))
    for got, was in zip(caches, pools):
        for g, w in zip(got, was):
            assert torch.equal(_bits(g.cpu()), _bits(TR.keep_ref(w, table, start, kv, kept, n_kept)))


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("H,d,page,n_caches", [(1, 64, 16, 1), (3, 128, 32, 3), (8, 64, 256, 1), (2, 128, 16, 64)])
def test_keep(dt, H, d, page, n_caches):
    for k, (sizes, kv) in enumerate([([1], [40]), ([16, 5, 0, 64], [16, 30, 9, 200]), ([40] * 20, [60 + i for i in range(20)]), ([300], [333])]):
        *case, n = _keep_case(sizes, kv, page, k)
        g = torch.Generator().manual_seed(k)
        pools = [tuple(torch.randn((n + i, H, page, d), generator=g).to(DT[dt]) for _ in range(2)) for i in range(n_caches if sum(kv) < 500 else 1)]
        _keep(pools, *case)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_keep_thins_out_long_requests(dt):
    for page in (16, 128):
        for sizes in ([5000], [4097, 1500, 7]):
            *case, n = _keep_case(sizes, sizes, page, 2)
            g = torch.Generator().manual_seed(1)
            _keep([tuple(torch.randn((n, 2, page, 64), generator=g).to(DT[dt]) for _ in range(2))], *case)


def test_keep_every_row_one_further():
    """Each row's place is the one that the row before has just left."""
    for n in (2, 65, 3000):
        table = np.random.default_rng(n).permutation(-(-n // 16))[None]
        g = torch.Generator().manual_seed(1)
        pools = [tuple(torch.randn((table.shape[1], 2, 16, 128), generator=g).to(torch.bfloat16) for _ in range(2))]
        _keep(pools, table, [0, n], [n], np.arange(1, n)[None], [n - 1])


@pytest.mark.parametrize("what", ["counts", "holes", "short", "not_rising", "no_rows"])
def test_keep_out_of_the_ordinary(what):
    page, g = 16, torch.Generator().manual_seed(3)
    table, start, kv, kept, n_kept, n = _keep_case([20, 64, 9], [100, 64, 30], page, 5, most=12)
    pools = [tuple(torch.randn((n, 2, page, 64), generator=g).to(torch.bfloat16) for _ in range(2))]
    if what == "counts":
        n_kept = [-3, 2 ** 31 - 1, 5]
        kept[1] = np.arange(1, 13)
    if what == "holes":
        table[0, 5], table[1, 1], table[2, 0] = -1, 10 ** 6, -2 ** 31
    if what == "short":
        table, kv = table[:, :4], [100, 50, 3]
    if what == "no_rows":
        start = [0, 20, 20, 9]
    if what == "not_rising":  # anything in the request's last tokens, nothing elsewhere
        kept[:, :] = np.random.default_rng(1).choice([-5, 0, 3, 63, 64, 2 ** 31 - 1, -2 ** 31], kept.shape)
        n_kept = [12, 12, 9]
        caches = [tuple(x.to(DEV) for x in p) for p in pools]
        fb.fedrag_paged_keep(caches, i32(table), i32(start), i32(kv), i32(kept), i32(n_kept))
        own = {(int(table[b, t // page]), t % page) for b in range(3) for t in range(kv[b] - int(start[b + 1] - start[b]), kv[b])}
        for got, was in zip(caches[0], pools[0]):
            same = (_bits(got.cpu()) == _bits(was)).all(-1).all(1)
            assert {(p, t) for p, t in (~same).nonzero().tolist()} <= own
        return
    _keep(pools, table, start, kv, kept, n_kept)


def test_keep_in_caches_that_take_turns():
    """Layers' pages side by side in one tensor: [n_pages, layers, 2, H, page, d]."""
    *case, n = _keep_case([30, 12], [50, 12], 16, 1)
    g = torch.Generator().manual_seed(2)
    x = torch.randn((n, 3, 2, 2, 16, 64), generator=g).to(torch.bfloat16)
    y = x.to(DEV)
    fb.fedrag_paged_keep([(y[:, i, 0], y[:, i, 1]) for i in range(3)], i32(case[0]), i32(case[1]), i32(case[2]), i32(case[3]), i32(case[4]))
    for i in range(3):
        for k in range(2):
            assert torch.equal(_bits(y[:, i, k].cpu()), _bits(TR.keep_ref(x[:, i, k].contiguous(), *case)))


# ----------------------------------------------------------------------------------------------- what goes
def _trim(kv, n_kept, table, free, count, page, start=None, in_place=False):
    k, fr, fc = i32(kv), i32(free), i32([count])
    kw = dict(lens_out=k, free_left=fc) if in_place else {}
    tb = i32(table)
    lens, left, flags = fb.fedrag_paged_trim(k, i32(n_kept), tb, fr, fc, page, q_start=None if start is None else i32(start), **kw)
    ref = TR.trim_ref(kv, n_kept, table, free, count, page, start)
    assert lens.tolist() == ref[0] and left.tolist() == [ref[2]] and flags.tolist() == [ref[3]]
    assert fr.tolist() == [int(x) for x in ref[1]]
    assert torch.equal(tb, i32(table))
    return ref


@pytest.mark.parametrize("B,page,top,tree", [(1, 16, 50, True), (7, 256, 900, True), (64, 16, 3000, True), (1025, 16, 40, True), (3, 32, 9000, False),
                                             (2300, 64, 130, False), (100, 16, 8000, False), (1, 16, 60000, True), (6, 16, 60000, False),
                                             (1500, 16, 90, False)])
def test_trim(B, page, top, tree):
    rng = np.random.default_rng(B)
    kv = rng.integers(1, top, B)
    n = rng.integers(0, np.minimum(kv, 64) + 1) if tree else None
    kept = rng.integers(0, n + 1) if tree else kv * (rng.random(B) < 0.5) * rng.integers(0, 2, B)
    columns = -(-int(kv.max()) // page) + 2
    table = rng.integers(0, 10 ** 9, (B, columns))
    free = rng.integers(0, 10 ** 9, 5 + int((-(-kv // page)).sum()))
    for in_place in (False, True):
        assert _trim(kv, kept, table, free, 5, page, TR.starts(n) if tree else None, in_place)[3] == 0


@pytest.mark.parametrize("what", ["full", "no_stack", "holes", "full_of_holes", "many", "lengths", "count_above", "count_below", "short", "no_requests", "no_columns"])
def test_trim_out_of_the_ordinary(what):
    rng = np.random.default_rng(4)
    B, page = 2500 if what == "many" else 300, 16
    kv, kept = rng.integers(1, 2000, B), rng.integers(0, 60, B)
    kept = np.minimum(kv, kept)
    table, free, count = rng.integers(0, 10 ** 6, (B, 130)), rng.integers(0, 10 ** 6, 30000 if B == 300 else 150000), 9
    if what == "full":
        free = free[:200]
    if what == "no_stack":
        free, count = free[:0], 0
    if what == "full_of_holes":
        free = free[:7003]
    if what in ("holes", "full_of_holes", "many"):
        table[rng.random(table.shape) < 0.3] = -1
        table[5:40] = -2 ** 31
    if what == "lengths":
        kv[[3, 7]], kept[[9, 11, 12]] = [-5, -2 ** 31], [-1, 2 ** 31 - 1, -2 ** 31]
    if what == "count_above":
        count = 30001
    if what == "count_below":
        count = -4
    if what == "short":
        table = table[:, :20].copy()
    if what == "no_columns":
        table = table[:, :0].copy()
    if what == "no_requests":
        kv, kept, table = kv[:0], kept[:0], table[:0]
    _trim(kv, kept, table, free, count, page)
    if what == "lengths":
        _trim(kv, kept, table, free, count, page, TR.starts(rng.integers(0, 50, B)))


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,G", [(1, 4), (3, 8), (6, 8)])
def test_many_short_requests(dt, n, G):
    """So many requests that shares hold several tiles each, none of them long enough to be cut: no partials are set aside (a table of
    256 tokens), and none are written."""
    B, Hkv = 900, 2
    rng = np.random.default_rng(n)
    kv = [n + int(rng.integers(0, 200)) for _ in range(B)]
    c = _attn_case([n] * B, kv, Hkv * G, Hkv, 64, 32, dt, seed=n)
    c["table"] = np.concatenate([c["table"], np.full((B, 8), -1)], 1)[:, :8]
    if dt != "f32":
        assert fb.fedrag_paged_tree_attn_workspace_bytes(B, Hkv * G, Hkv, 64, DT[dt], n * B, 8, 32, n) == 0
    O, lse = _attn(c, check=False)
    pick = sorted(rng.choice(B, 12, replace=False))
    rows = np.concatenate([np.arange(c["start"][b], c["start"][b + 1]) for b in pick])
    ref = TR.attn_ref(c["Q"][:, rows], c["Kp"], c["Vp"], c["table"][pick], n * np.arange(13), [kv[b] for b in pick], c["mask"][rows], 64 ** -0.5)
    R.check_attn(O[:, :, rows], lse[:, :, rows], ref, FILL)


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f16", 64)])
def test_short_units(dt, d):
    """17 to 32 rows over 257 to 2048 tokens, where keys are cut into shorter units; around those bounds, beside requests of none and of one unit."""
    for sizes, kv in (([6], [257]), ([6], [2048]), ([6], [2049]), ([8, 5, 0, 7], [129, 128, 300, 1000]), ([8, 8, 8], [8, 384, 900]), ([5, 8], [500, 700]),
                      ([8], [256])):
        _attn(_attn_case(sizes, kv, 8, 2, d, 16, dt, seed=sum(kv), columns_more=0), what=(sizes, kv))


def test_pages_beyond_4_gib():
    """Attention, and rows moved, in pages whose bytes are numbered beyond 2^32."""
    H, page, d, n = 8, 256, 128, 9000
    K, V = (torch.zeros((n, H, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))  # 4.7 GB each
    table = np.array([[8999, 3, 8500, 8998]])
    g = torch.Generator().manual_seed(1)
    small = [torch.randn((4, H, page, d), generator=g).to(torch.bfloat16) for _ in range(2)]
    for big, x in zip((K, V), small):
        big[torch.tensor(table[0]).to(DEV)] = x.to(DEV)
    Q, up = torch.randn((8, 9, d), generator=g).to(torch.bfloat16), TR.trees(np.random.default_rng(1), [9])
    mask = TR.signed(TR.map_ref(up, [0, 9], [1000], 1, 9)[0])
    O, lse = fb.fedrag_paged_tree_attn(Q.to(DEV), K, V, i32(table), i32([0, 9]), i32([1000]), torch.from_numpy(mask).to(DEV), 9)
    R.check_attn(O, lse, TR.attn_ref(Q, *small, np.arange(4)[None], [0, 9], [1000], mask, d ** -0.5), FILL)
    kept = np.array([[0, 2, 5, 6, 8]])
    fb.fedrag_paged_keep([(K, V)], i32(table), i32([0, 9]), i32([1000]), i32(kept), i32([5]))
    for big, x in zip((K, V), small):
        want = TR.keep_ref(x, np.arange(4)[None], [0, 9], [1000], kept, [5])
        assert torch.equal(_bits(big[torch.tensor(table[0]).to(DEV)].cpu()), _bits(want))
        assert not big[4:8400].any()


def test_refusals_of_tensors():
    """What the binding finds wrong with tensors on the device."""
    i, f = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.float64, device=DEV)
    pages, p = torch.zeros((3, 1, 16, 64), device=DEV), torch.ones((4, 10), device=DEV)
    table, kept, mask = i.view(2, 2), i.view(2, 2), torch.zeros((4, 1), dtype=torch.int64, device=DEV)
    Q = torch.zeros((1, 4, 64), device=DEV)
    attn = lambda **kw: fb.fedrag_paged_tree_attn(*{**dict(Q=Q, K=pages, V=pages.clone(), t=table, s=i[:3], kv=i[:2], m=mask), **kw}.values())  # noqa: E731
    attn()
    verify = lambda **kw: fb.fedrag_tree_verify(**{**dict(target=p, tokens=i, parents=i, q_start=i[:2], u=f, u_next=f[:1]), **kw})  # noqa: E731
    verify()
    for call in (lambda: attn(m=mask[:3]), lambda: attn(m=mask.int()), lambda: attn(m=mask[:, 0]), lambda: attn(Q=Q.half()), lambda: attn(s=i[:2]),
                 lambda: attn(t=i), lambda: attn(K=pages.expand(3, 1, 16, 64)[:1].expand(3, 1, 16, 64)), lambda: verify(u=f.float()),
                 lambda: verify(draft=p.half()), lambda: verify(draft=p[:3]), lambda: verify(target=p.double()), lambda: verify(tokens=i[:3]),
                 lambda: verify(target=p.t().contiguous().t()), lambda: verify(target=p[:1].expand(4, 10)), lambda: verify(kept=kept, max_kept=3),
                 lambda: fb.fedrag_tree_map(i, i[:3], i[:2], 0), lambda: fb.fedrag_tree_map(i.long(), i[:3], i[:2], 1),
                 lambda: fb.fedrag_tree_map(i, i[:2], i[:2], 1), lambda: fb.fedrag_paged_keep([(pages, pages.half())], table, i[:3], i[:2], kept, i[:2]),
                 lambda: fb.fedrag_paged_keep([(pages, pages.clone()), (pages[:, :, :, :32], pages[:, :, :, :32])], table, i[:3], i[:2], kept, i[:2]),
                 lambda: fb.fedrag_paged_keep([(pages, pages.clone(), pages)], table, i[:3], i[:2], kept, i[:2]),
                 lambda: fb.fedrag_paged_keep([(pages, pages.clone())], table, i[:3], i[:2], kept, i[:3]),
                 lambda: fb.fedrag_paged_trim(i[:2], i[:2], table, i.long(), i[:1], 16), lambda: fb.fedrag_paged_trim(i[:2], i[:3], table, i, i[:1], 16)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: fb.fedrag_paged_keep([(pages, pages)], table, i[:3], i[:2], kept, i[:2]), lambda: fb.fedrag_tree_map(i, i[:3], i[:2], 65),
                 lambda: fb.fedrag_paged_trim(i[:2], i[:2], table, i, i[:1], 24)):
        with pytest.raises(fb.FedragError):
            call()
