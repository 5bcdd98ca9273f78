"""The paged calls as a serving node uses them, together and with the calls they stand beside: a Compute Node's cache of scrambled
contexts, an Inquirer's growing cache of its own tokens, prompts in one step and decoded tokens in the next ones, recorded and
replayed; and calls that run at once."""
import numpy as np
import pytest
import torch

import paged_ref as R
from paper_2605_25716_amd import binding as fb
from paper_2605_25716_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int64).astype(np.int32)).to(DEV)


class Node:
    """A cache of n_pages pages and the state that fedrag_paged_map advances."""

    def __init__(self, B, n_pages, columns, Hkv, page, d, dtype, seed):
        g = torch.Generator().manual_seed(seed)
        self.K, self.V = (torch.full((n_pages, Hkv, page, d), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
        self.table = torch.full((B, columns), -1, dtype=torch.int32, device=DEV)
        self.free = torch.randperm(n_pages, generator=g).to(torch.int32).to(DEV)
        self.count, self.lens, self.page = i32([n_pages]), i32([0] * B), page

    def step(self, new, T, K, V):
        """Plans a step of `new` rows a request in place and writes its rows; (q_start, flags)"""
        q_start, _, slots, _, _, flags = fb.fedrag_paged_map(self.lens, new, self.table, self.free, self.count, self.page, T,
                                                             kv_lens=self.lens, free_left=self.count)
        fb.fedrag_paged_write(K, V, slots, self.K, self.V)
        return q_start, flags


def test_requests_over_two_nodes():
    """Prompts, then decoded tokens by a recorded step, against attention over each request's context and own tokens in 64 bits.
    fp32 storage: products with orthogonal keys are within some 3e-6 of their size, logits of up to 8 within 3e-5, probabilities
    within twice that and the outputs, norm-wise, within 1e-4."""
    B, Hq, Hkv, d, page, dtype = 3, 8, 2, 64, 16, torch.float32
    ctx, prompt, steps = [100, 37, 300], [20, 5, 33], 4
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    keys = W.make_keys(Hkv, d, sum(prompt), 300, 1, seed=5, dtype=dtype)
    phi = {k: getattr(keys, k).to(DEV) for k in ("phi_q", "phi_k", "phi_v", "phi_v_inv")}

    # the Context Owners' part, once: each context scrambled in its own order, its rows into the Compute Node's pages
    remote = Node(B, 40, 24, Hkv, page, d, dtype, 1)
    Kc, Vc = [rnd(1, Hkv, n, d) for n in ctx], [rnd(1, Hkv, n, d) for n in ctx]
    scr = [fb.fedrag_scramble_kv(k.to(DEV), v.to(DEV), phi["phi_k"], phi["phi_v"], torch.randperm(n, generator=g).to(torch.int32).to(DEV))
           for k, v, n in zip(Kc, Vc, ctx)]
    T = sum(ctx)
    _, flags = remote.step(i32(ctx), T, torch.cat([s[0] for s in scr], 2), torch.cat([s[1] for s in scr], 2))
    assert int(flags) == 0

    local = Node(B, 30, 9, Hkv, page, d, dtype, 2)
    seen_k, seen_v = [[] for _ in range(B)], [[] for _ in range(B)]

    def layer(new, T, Q, K, V, max_q):
        """One layer's attention of a step: the Inquirer's own part, the Compute Node's, and their aggregation."""
        q_start, flags = local.step(new, T, K, V)
        own = fb.fedrag_paged_attn(Q, local.K, local.V, local.table, q_start, local.lens, max_q, causal=True)
        far = fb.fedrag_paged_attn(fb.fedrag_scramble_q(Q, phi["phi_q"]), remote.K, remote.V, remote.table, q_start, remote.lens, max_q,
                                   causal=False)
        O, lse = fb.fedrag_unscramble_merge(*far, phi["phi_v_inv"], None, *own, n_kv_heads=Hkv)
        return O, lse, flags

    def check(O, new, Q, K, V, what):
        at = 0
        for b, n in enumerate(new):
            seen_k[b].append(K[0, :, at:at + n])
            seen_v[b].append(V[0, :, at:at + n])
            k, v = (torch.cat([c[b][0]] + s[b], 1).double().numpy() for c, s in ((Kc, seen_k), (Vc, seen_v)))
            for h in range(Hq):
                for i in range(n):
                    m = k.shape[1] - n + i + 1
                    x = k[h // (Hq // Hkv), :m] @ Q[0, h, at + i].double().numpy() * d ** -0.5
                    p = np.exp(x - x.max())
                    want = p @ v[h // (Hq // Hkv), :m] / p.sum()
                    got = O[0, h, at + i].double().cpu().numpy()
                    assert np.abs(got - want).max() <= 1e-4 * np.abs(want).max(), (what, b, h, i)
            at += n

    T = sum(prompt)
    Q, K, V = rnd(1, Hq, T, d), rnd(1, Hkv, T, d), rnd(1, Hkv, T, d)
    O, _, flags = layer(i32(prompt), T, Q.to(DEV), K.to(DEV), V.to(DEV), max(prompt))
    assert int(flags) == 0
    check(O, prompt, Q, K, V, "prompt")

    # decoded tokens: the step is recorded once; request 1 stops after two of them
    new, Qd, Kd, Vd = i32([1] * B), torch.empty((1, Hq, B, d), device=DEV), torch.empty((1, Hkv, B, d), device=DEV), torch.empty((1, Hkv, B, d), device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        O, _, flags = layer(new, B, Qd, Kd, Vd, 1)
    for s in range(steps):
        n = [1, 1 if s < 2 else 0, 1]
        T = sum(n)
        Q, K, V = rnd(1, Hq, T, d), rnd(1, Hkv, T, d), rnd(1, Hkv, T, d)
        new.copy_(i32(n))
        for dst, src in ((Qd, Q), (Kd, K), (Vd, V)):
            dst.zero_()
            dst[:, :, :T] = src.to(DEV)
        if s == 2:  # an eager step between the replays
            got, _, fl = layer(new, B, Qd, Kd, Vd, 1)
        else:
            graph.replay()
            got, fl = O, flags
        torch.cuda.synchronize()
        assert int(fl) == 0
        check(got, n, Q, K, V, f"token {s}")
    assert local.lens.tolist() == [20 + steps, 7, 33 + steps]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_recorded_attention_replays(dt):
    """A recorded call with runs and partials, replayed with other work between, gives the eager call's bits every time; a second
    recorded call has scratch of its own."""
    Hq, Hkv, d, page = 8, 2, 128, 32
    g = torch.Generator(device=DEV).manual_seed(1)
    q, kv = [1, 40, 1], [2500, 1300, 700]
    n_pages = sum(-(-n // page) for n in kv)
    Kp, Vp = (torch.randn((n_pages, Hkv, page, d), generator=g, device=DEV).to(dt) for _ in range(2))
    table = np.full((3, 80), -1)
    at = 0
    for b, n in enumerate(kv):
        table[b, :-(-n // page)] = np.arange(at, at - (-n // page))
        at += -(-n // page)
    args = lambda Q: (Q, Kp, Vp, i32(table), i32([0, 1, 41, 42]), i32(kv), 40)  # noqa: E731
    calls = []
    for _ in range(2):
        a = args(torch.randn((Hq, 42, d), generator=g, device=DEV).to(dt))
        want = fb.fedrag_paged_attn(*a)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            got = fb.fedrag_paged_attn(*a)
        calls.append((graph, got, want, a))
    for k in range(4):
        side = torch.cuda.Stream()
        for (graph, got, _, a), stream in zip(calls, (torch.cuda.current_stream(), side)):
            for x in got:
                x.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                graph.replay()  # both at once
        fb.fedrag_paged_attn(*calls[k % 2][3])
        torch.cuda.synchronize()
        for _, got, want, _ in calls:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), k


def test_calls_on_two_streams():
    """Calls on another stream than the default one, at the same time, with scratch of their own."""
    Hq, Hkv, d, page = 8, 2, 64, 16
    Q, Kp, Vp = (torch.randn(s, device=DEV).to(torch.float16) for s in ((Hq, 4, d), (400, Hkv, page, d), (400, Hkv, page, d)))
    table = torch.randperm(400).to(torch.int32).view(4, 100).to(DEV)
    args = (Q, Kp, Vp, table, i32([0, 1, 2, 3, 4]), i32([1600, 900, 20, 1111]), 1)
    want = fb.fedrag_paged_attn(*args)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for k in range(6):
        with torch.cuda.stream(streams[k % 2]):
            outs.append(fb.fedrag_paged_attn(*args))
    torch.cuda.synchronize()
    for O, lse in outs:
        assert torch.equal(O, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_thousands_of_requests(dt):
    """More requests than a lane has in one look (64 lanes, 64 each), most of them short, one long, some empty."""
    B, Hq, Hkv, d, page = 4200, 2, 1, 64, 16
    rng = np.random.default_rng(1)
    q = (rng.random(B) < 0.9).astype(np.int64)
    kv = rng.integers(0, 30, B)
    q[4100], kv[4100], q[17], kv[17], q[4199], kv[4199] = 30, 2000, 40, 60, 1, 900
    n_pages = int(sum(-(-n // page) for n in kv))
    g = torch.Generator().manual_seed(2)
    table = np.full((B, 125), -1)
    at = 0
    for b, n in enumerate(kv):
        table[b, :-(-n // page)] = np.arange(at, at - (-n // page))
        at += -(-n // page)
    Q, Kp, Vp = torch.randn((Hq, int(q.sum()), d), generator=g).to(dt), torch.randn((n_pages, Hkv, page, d), generator=g).to(dt), \
        torch.randn((n_pages, Hkv, page, d), generator=g).to(dt)
    start = np.concatenate([[0], np.cumsum(q)])
    ref = R.attn_ref(Q, Kp, Vp, table, start, kv, True, d ** -0.5)
    for max_q in (40, 1):
        O = torch.full((1,) + tuple(Q.shape), 7.0, device=DEV)
        lse = torch.full((1, Hq, Q.shape[1]), 7.0, device=DEV)
        fb.fedrag_paged_attn(Q.to(DEV), Kp.to(DEV), Vp.to(DEV), i32(table), i32(start), i32(kv), max_q, O_part=O, lse=lse)
        R.check_attn(O, lse, ref, 7.0, f"max_q {max_q}")


def test_binding_refusals_on_the_device():
    Q, Kp = torch.zeros((4, 3, 64), device=DEV), torch.zeros((5, 2, 16, 64), device=DEV)
    ok = dict(Q=Q, K_pages=Kp, V_pages=Kp.clone(), block_table=i32([[0, 1]]), q_start=i32([0, 3]), kv_lens=i32([9]))
    fb.fedrag_paged_attn(**ok)
    for name, bad in (("Q", Q.half()), ("Q", Q[..., ::2]), ("Q", Q[:, :, :32]), ("Q", Q[0]), ("Q", Q.cpu()), ("V_pages", Kp[:4]), ("V_pages", Kp.half()),
                      ("V_pages", Kp.cpu()), ("K_pages", Kp[:, :, ::2]), ("block_table", i32([0, 1])), ("block_table", i32([[0, 1]]).long()),
                      ("q_start", i32([0])), ("q_start", i32([0, 3]).float()), ("q_start", torch.tensor([0, 3], dtype=torch.int32)),
                      ("kv_lens", i32([9, 9])), ("O_part", torch.zeros((1, 4, 2, 64), device=DEV)), ("lse", torch.zeros(12, device=DEV).half()),
                      ("O_part", torch.zeros((1, 4, 64, 3), device=DEV).transpose(2, 3))):
        with pytest.raises(ValueError):
            fb.fedrag_paged_attn(**{**ok, name: bad})
    for kw, status in ((dict(max_q_len=-1), fb.ERR_SHAPE), (dict(softmax_scale=0.0), fb.ERR_SHAPE), (dict(O_part=Kp), fb.ERR_ALIAS),
                       (dict(K_pages=Kp.view(10, 2, 8, 64), V_pages=Kp.view(10, 2, 8, 64)), fb.ERR_UNSUPPORTED)):
        with pytest.raises(fb.FedragError) as e:
            fb.fedrag_paged_attn(**{**ok, **kw})
        assert e.value.status == status
    rows = torch.zeros((2, 3, 64), device=DEV)
    for K, V, slots in ((rows.half(), rows, 3), (rows, rows[:, :2], 3), (rows[:1], rows[:1], 3), (rows, rows, 2)):
        with pytest.raises(ValueError):
            fb.fedrag_paged_write(K, V, torch.zeros(slots, dtype=torch.int64, device=DEV), Kp, Kp.clone())
    with pytest.raises(fb.FedragError):
        fb.fedrag_paged_write(rows, rows, torch.zeros(3, dtype=torch.int64, device=DEV), Kp, Kp)
    with pytest.raises(TypeError):
        fb.fedrag_paged_attn(**ok, max_q_len=1.5)


def test_expanded_pools_are_refused():
    """One page under many ids: there is no memory behind the others."""
    Q, rows, page = torch.zeros((4, 3, 64), device=DEV), torch.zeros((2, 3, 64), device=DEV), torch.zeros((1, 2, 16, 64), device=DEV)
    K, V = page.expand(5, 2, 16, 64), page.clone().expand(5, 2, 16, 64)
    with pytest.raises(ValueError):
        fb.fedrag_paged_attn(Q, K, V, i32([[0, 1]]), i32([0, 3]), i32([9]))
    with pytest.raises(ValueError):
        fb.fedrag_paged_write(rows, rows, torch.zeros(3, dtype=torch.int64, device=DEV), K, V)
