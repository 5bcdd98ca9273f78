"""Drafted steps as an Inquirer takes them: planned, written, attended to in every layer, verified, what stays moved together, what
does not given back; recorded and replayed with eager steps between; beside a Compute Node's part; and calls that run at once."""
import numpy as np
import pytest
import torch

import paged_ref as R
import tree_ref as TR
from paper_2605_25716_amd import binding as fb
from paper_2605_25716_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int64).astype(np.int32)).to(DEV)


@pytest.mark.parametrize("dt,with_draft", [(torch.float32, True), (torch.bfloat16, False)])
def test_drafted_steps_recorded_and_replayed(dt, with_draft):
    B, layers, Hq, Hkv, d, page, V, most = 3, 2, 8, 2, 64, 16, 300, 5
    n_pages, columns, T, words = 40, 12, 30, 1
    g = torch.Generator().manual_seed(5)
    rng = np.random.default_rng(5)
    rnd = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    pools = [tuple(torch.full((n_pages, Hkv, page, d), float("nan"), dtype=dt, device=DEV) for _ in range(2)) for _ in range(layers)]
    table = torch.full((B, columns), -1, dtype=torch.int32, device=DEV)
    free, count, lens = i32(rng.permutation(n_pages)), i32([n_pages]), i32([0] * B)
    # what the steps take, in place
    new, up, tokens = i32([0] * B), i32([-1] * T), i32([0] * T)
    Q = torch.zeros((layers, 1, Hq, T, d), dtype=dt, device=DEV)
    K, Vv = (torch.zeros((layers, 1, Hkv, T, d), dtype=dt, device=DEV) for _ in range(2))
    p, q = (torch.zeros((T, V), device=DEV) for _ in range(2))
    u, u_next = torch.zeros(T, dtype=torch.float64, device=DEV), torch.zeros(B, dtype=torch.float64, device=DEV)

    def step():
        q_start, kv, slots, _, _, flags = fb.fedrag_paged_map(lens, new, table, free, count, page, T, free_left=count)
        mask, positions, bad = fb.fedrag_tree_map(up, q_start, kv, words)
        out = []
        for i in range(layers):
            fb.fedrag_paged_write(K[i], Vv[i], slots, *pools[i])
            out.append(fb.fedrag_paged_tree_attn(Q[i], *pools[i], table, q_start, kv, mask, 12))
        kept, n_kept, nxt = fb.fedrag_tree_verify(p, tokens, up, q_start, u, u_next, draft=q if with_draft else None, max_kept=most)
        fb.fedrag_paged_keep(pools, table, q_start, kv, kept, n_kept)
        _, _, trimmed = fb.fedrag_paged_trim(kv, n_kept, table, free, count, page, q_start=q_start, lens_out=lens, free_left=count)
        return out, q_start, kv, mask, positions, bad, kept, n_kept, nxt, flags, trimmed

    history = [[[] for _ in range(B)] for _ in range(2 * layers)]  # the K, V rows that each request has kept, in order
    graph, recorded = None, None
    for s in range(7):
        n = rng.integers(1, 11, B)
        n[s % B] = 0 if s == 3 else n[s % B]  # a request that sits out
        start = TR.starts(n)
        parents = np.full(T, -1)
        parents[:start[-1]] = TR.trees(rng, n, "tree" if s % 2 else "chain")
        host = dict(Q=rnd(*Q.shape).to(dt), K=rnd(*K.shape).to(dt), V=rnd(*Vv.shape).to(dt))
        logits = 2.0 * rnd(T, V)
        hp, hq = torch.softmax(logits, -1), torch.softmax(logits + 0.4 * rnd(T, V), -1)
        owner = np.repeat(start[:-1], n)
        above = np.zeros(T, np.int64)
        above[:start[-1]] = owner + np.maximum(parents[:start[-1]], 0)
        tok = torch.multinomial(hq[above], 1, generator=g)[:, 0] if with_draft else hp[above].topk(3, -1)[1][np.arange(T), rng.integers(0, 3, T)]
        hu, hn = rng.random(T), rng.random(B)
        if graph is None and s == 2:  # (the first steps are eager, as a program's are)
            graph = torch.cuda.CUDAGraph()
            state = [x.clone() for x in (table, free, count, lens, *[y for pool in pools for y in pool])]
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                recorded = step()
            for x, y in zip((table, free, count, lens, *[y for pool in pools for y in pool]), state):
                assert torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float()))  # recording runs nothing
        for dst, src in ((new, i32(n)), (up, i32(parents)), (tokens, i32(tok.numpy())), (Q, host["Q"]), (K, host["K"]), (Vv, host["V"]), (p, hp),
                         (q, hq), (u, torch.from_numpy(hu)), (u_next, torch.from_numpy(hn))):
            dst.copy_(src)
        before = lens.cpu().numpy().copy()
        if graph is None or s == 4:
            got = step()
        else:
            graph.replay()
            got = recorded
        torch.cuda.synchronize()
        out, q_start, kv, mask, positions, bad, kept, n_kept, nxt, flags, trimmed = got
        assert q_start.tolist() == start.tolist() and kv.tolist() == (before + n).tolist() and int(flags) == 0 and int(trimmed) == 0
        masks, pos, bad_ref = TR.map_ref(parents, start, before + n, words, T)
        assert mask.tolist() == TR.signed(masks).tolist() and positions.tolist() == pos and bad.tolist() == bad_ref == [0] * B
        # attention: against the rows as the requests have them, not as the pages hold them
        for i in range(layers):
            for b in range(B):
                rows = slice(int(start[b]), int(start[b + 1]))
                if n[b] == 0:
                    continue
                k, v = (torch.stack(history[2 * i + j][b] + list(x[i, 0, :, rows].transpose(0, 1))) for j, x in enumerate((host["K"], host["V"])))
                P1 = -(-len(k) // page)
                pad = torch.zeros((P1 * page - len(k), Hkv, d), dtype=dt)
                kp, vp = (torch.cat([x, pad]).view(P1, page, Hkv, d).transpose(1, 2) for x in (k, v))
                ref = TR.attn_ref(host["Q"][i, 0][:, rows], kp, vp, np.arange(P1)[None], [0, n[b]], [len(k)], TR.signed(masks[rows]), d ** -0.5)
                O, lse = out[i]
                R.check_attn(O[:, :, rows], lse[:, :, rows], ref, None, f"step {s} layer {i} request {b}")
        ref = TR.verify_ref(hp, hq if with_draft else None, tok.numpy(), parents, start, hu, hn, most)
        for x, y in zip((kept, n_kept, nxt), ref):
            assert x.tolist() == y.tolist(), f"step {s}"
        assert lens.tolist() == (before + ref[1]).tolist()
        for i in range(layers):
            for j, x in enumerate((host["K"], host["V"])):
                for b in range(B):
                    history[2 * i + j][b] += [x[i, 0, :, start[b] + int(r)] for r in ref[0][b, :ref[1][b]]]
        # the pages hold just that, and every page is a request's or free, once
        tb, used = table.cpu().numpy(), []
        for b in range(B):
            L = int(lens[b])
            ids = tb[b, :-(-L // page)]
            used += ids.tolist()
            for i in range(layers):
                for j in range(2):
                    rows = pools[i][j].cpu()[ids.astype(np.int64)].transpose(1, 2).reshape(-1, Hkv, d)[:L]
                    assert torch.equal(rows, torch.stack(history[2 * i + j][b]) if L else rows)
        assert sorted(used + free[:int(count)].tolist()) == list(range(n_pages))
    assert max(len(h) for h in history[0]) > (page if with_draft else 5)  # (the steps have come some way; few drafts that were not drawn stay)


def test_drafts_over_two_nodes():
    """One layer's attention of a drafted step: the Inquirer's own tokens by the tree, the Compute Node's scrambled context whole, and
    their aggregation, against attention over both in 64 bits (fp32 storage: within 1e-4, norm-wise, as for undrafted tokens)."""
    B, Hq, Hkv, d, page = 2, 8, 2, 64, 16
    ctx, had, sizes = [90, 200], [21, 5], [7, 12]
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    keys = W.make_keys(Hkv, d, sum(sizes), 300, 1, seed=5, dtype=torch.float32)
    phi = {k: getattr(keys, k).to(DEV) for k in ("phi_q", "phi_k", "phi_v", "phi_v_inv")}
    T, start = sum(sizes), TR.starts(sizes)
    up = TR.trees(np.random.default_rng(3), sizes)

    def cache(rows):
        """Requests' rows [1, Hkv, L, d] in pages: (pages of K and of V, table)"""
        lens = [k.shape[2] for k, _ in rows]
        need = [-(-n // page) for n in lens]
        pools = [torch.zeros((sum(need), Hkv, page, d), device=DEV) for _ in range(2)]
        table, free, count = torch.full((B, max(need)), -1, dtype=torch.int32, device=DEV), i32(range(sum(need))), i32([sum(need)])
        _, kv, slots, _, _, flags = fb.fedrag_paged_map(i32([0] * B), i32(lens), table, free, count, page, sum(lens))
        fb.fedrag_paged_write(torch.cat([k for k, _ in rows], 2), torch.cat([v for _, v in rows], 2), slots, *pools)
        assert int(flags) == 0
        return pools, table, kv

    Kc, Vc = [rnd(1, Hkv, n, d) for n in ctx], [rnd(1, Hkv, n, d) for n in ctx]
    far = cache([fb.fedrag_scramble_kv(k.to(DEV), v.to(DEV), phi["phi_k"], phi["phi_v"], torch.randperm(n, generator=g).to(torch.int32).to(DEV))
                 for k, v, n in zip(Kc, Vc, ctx)])
    Kl, Vl = [rnd(1, Hkv, h + n, d) for h, n in zip(had, sizes)], [rnd(1, Hkv, h + n, d) for h, n in zip(had, sizes)]
    own = cache([(k.to(DEV), v.to(DEV)) for k, v in zip(Kl, Vl)])
    Q = rnd(1, Hq, T, d)
    q_start = i32(start)
    mask, _, _ = fb.fedrag_tree_map(i32(up), q_start, own[2], 1)
    near = fb.fedrag_paged_tree_attn(Q.to(DEV), *own[0], own[1], q_start, own[2], mask, max(sizes))
    there = fb.fedrag_paged_attn(fb.fedrag_scramble_q(Q.to(DEV), phi["phi_q"]), *far[0], far[1], q_start, far[2], max(sizes), causal=False)
    O, _ = fb.fedrag_unscramble_merge(*there, phi["phi_v_inv"], None, *near, n_kv_heads=Hkv)
    bits = TR.map_ref(up, start, [h + n for h, n in zip(had, sizes)], 1, T)[0]
    for b in range(B):
        for i in range(sizes[b]):
            sees = [*range(had[b]), *[had[b] + j for j in range(sizes[b]) if bits[start[b] + i][0] >> j & 1]]
            for h in range(Hq):
                k = torch.cat([Kc[b][0, h // 4], Kl[b][0, h // 4, sees]]).double().numpy()
                v = torch.cat([Vc[b][0, h // 4], Vl[b][0, h // 4, sees]]).double().numpy()
                x = k @ Q[0, h, start[b] + i].double().numpy() * d ** -0.5
                e = np.exp(x - x.max())
                want, got = e @ v / e.sum(), O[0, h, start[b] + i].double().cpu().numpy()
                assert np.abs(got - want).max() <= 1e-4 * np.abs(want).max(), (b, i, h)


def _attn_args(seed, dt=torch.bfloat16, sizes=(1, 12, 70), kv=(2500, 5300, 900)):
    g = torch.Generator(device=DEV).manual_seed(seed)
    need = [-(-n // 32) for n in kv]
    table = np.full((len(kv), max(need) + 1), -1)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = np.arange(at, at + n)
        at += n
    Kp, Vp = (torch.randn((at, 2, 32, 128), generator=g, device=DEV).to(dt) for _ in range(2))
    up, T = TR.trees(np.random.default_rng(seed), sizes), sum(sizes)
    mask, _, _ = fb.fedrag_tree_map(i32(up), i32(TR.starts(sizes)), i32(kv), 2)
    return torch.randn((8, T, 128), generator=g, device=DEV).to(dt), Kp, Vp, i32(table), i32(TR.starts(sizes)), i32(kv), mask, max(sizes)


FORMS = [(1, 2, 1), (1, 7, 4), (12, 3, 16), (1, 12, 70), (70, 70, 70)]


@pytest.mark.parametrize("sizes", FORMS)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_recorded_attention_replays(dt, sizes):
    """Runs, shares and partials of a recorded call, replayed with other work between: the eager call's bits every time, and a second
    recorded call has scratch of its own."""
    calls = []
    for seed in (1, 2):
        a = _attn_args(seed, dt, sizes)
        want = fb.fedrag_paged_tree_attn(*a)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            got = fb.fedrag_paged_tree_attn(*a)
        calls.append((graph, got, want, a))
    for k in range(4):
        for graph, got, want, a in calls:
            got[0].zero_()
            got[1].zero_()
            graph.replay()
            if k % 2:
                fb.fedrag_paged_tree_attn(*a)  # eager, with scratch of its own
        torch.cuda.synchronize()
        for _, got, want, _ in calls:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_calls_at_once():
    """Two streams, each with its own step, against the same calls one after the other."""
    V = 9000
    g = torch.Generator(device=DEV).manual_seed(1)
    work = []
    for seed in (3, 4):
        a = _attn_args(seed)
        T = a[0].shape[1]
        up = i32(TR.trees(np.random.default_rng(seed), (1, 12, 70)))
        p, q = (torch.softmax(2 * torch.randn((T, V), generator=g, device=DEV), -1) for _ in range(2))
        tokens = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
        u, un = (torch.rand(n, generator=g, device=DEV, dtype=torch.float64) for n in (T, 3))
        work.append((a, (p, tokens, up, a[4], u, un), q))

    def run(a, v, q):
        O, lse = fb.fedrag_paged_tree_attn(*a)
        out = fb.fedrag_tree_verify(*v, draft=q, max_kept=9)
        pages = (a[1].clone(), a[2].clone())
        fb.fedrag_paged_keep([pages], a[3], a[4], a[5], out[0], out[1])
        free, count = torch.full((500,), -1, dtype=torch.int32, device=DEV), i32([3])
        return [O, lse, *out, *pages, free, *fb.fedrag_paged_trim(a[5], out[1], a[3], free, count, 32, q_start=a[4])]

    want = [run(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(3):
        got = []
        for s, w in zip(streams, work):
            with torch.cuda.stream(s):
                got.append(run(*w))
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert all(torch.equal(i, j) for i, j in zip(x, y))


@pytest.mark.parametrize("V", [5000, 40000])
def test_recorded_verification_replays(V):
    """One launch, and rounds over a workspace that holds anything, replayed with new inputs in place."""
    rng = np.random.default_rng(1)
    sizes = [9, 30, 4]
    start, T = TR.starts(sizes), sum(sizes)
    up = TR.trees(rng, sizes)
    g = torch.Generator().manual_seed(1)
    draw = lambda: [torch.softmax(2 * torch.randn((T, V), generator=g), -1) for _ in range(2)]  # noqa: E731
    p, q = (x.to(DEV) for x in draw())
    tokens, u, un = i32([0] * T), torch.zeros(T, dtype=torch.float64, device=DEV), torch.zeros(3, dtype=torch.float64, device=DEV)
    ws = torch.full((fb.fedrag_tree_verify_workspace_bytes(3, V, torch.float32),), 255, dtype=torch.uint8, device=DEV)
    args = (p, tokens, i32(up), i32(start), u, un)
    fb.fedrag_tree_verify(*args, draft=q, max_kept=7, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = fb.fedrag_tree_verify(*args, draft=q, max_kept=7, workspace=ws)
    for k in range(5):
        hp, hq = draw()
        ht, hu, hn = rng.integers(0, 40, T), rng.random(T) ** (k + 1), rng.random(3)
        hp[:, :40] *= 50
        hp /= hp.sum(-1, keepdim=True)
        for dst, src in ((p, hp), (q, hq), (tokens, i32(ht)), (u, torch.from_numpy(hu)), (un, torch.from_numpy(hn))):
            dst.copy_(src)
        ws.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, TR.verify_ref(hp, hq, ht, up, start, hu, hn, 7)):
            assert x.tolist() == y.tolist(), k
