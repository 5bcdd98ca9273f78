"""A drafted step over the paged cache: a tree of tokens attended to, verified, and what was accepted kept.  The work whose speed counts.

Kinds of cases (key "kind"):
  tree_map   ancestor masks and positions of the drafted rows, from their parents.
  tree_attn  attention of the drafted rows over the pages: a row sees what the request had before and its own ancestors.
  verify     the walk from the root: accepted rows and the next token, from the target's probabilities (and the draft's) and given
             random numbers.
  keep       the accepted rows' K, V moved to the front of the request's drafted tokens, all layers in one call.
  trim       the lengths that are left, and the pages no longer needed back on the stack of free ones.

"q" and "kv" are the requests' drafted rows and their keys (the drafted rows among them), comma separated.  Row 0 of a request is its
last token, which is decided; the others are drafts, in order of depth.  Activations are N(0,1) with 1 % of the (head, channel) axis
scaled by 20; probabilities are a softmax over logits of a spread of about 2.5 by which a few tokens carry most of the weight, and the draft's logits
are the target's and noise.  Pages are handed out in random order, as after a while of serving.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LLAMA8B = dict(Hq=32, Hkv=8, d=128)
UNIT = 2.0 ** 43  # weights of tokens are whole numbers of 2^-43


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _spread(n, lo, hi):
    """n lengths from hi down to lo, evenly over their logarithm, none of them round."""
    if n == 1:
        return [hi]
    return [max(1, int(round(hi * (lo / hi) ** (i / (n - 1)))) - (i % 3)) for i in range(n)]


def listed():
    return [
        # the tree of one request: what a step's bookkeeping costs at the least
        dict(name="map_one", kind="tree_map", q="8", kv="801", words=1, T=8),
        # a step of 256 requests, some with large trees, some not drafting, rows padded to a round number
        dict(name="map_many", kind="tree_map", q=_text([[1, 64, 17, 33][i % 4] for i in range(256)]), kv=_text(_spread(256, 70, 16000)), words=1,
             T=7424),
        # a short request with a few drafts: latency
        dict(name="tree_short", kind="tree_attn", q="6", kv="198", words=1, page=16, dtype="bf16", pad=0, **LLAMA8B),
        # 32 requests of very unequal lengths with 16 nodes each: bound by the keys' bytes
        dict(name="tree_ragged", kind="tree_attn", q=_text([16] * 32), kv=_text(_spread(32, 1000, 32768)), words=1, page=16, dtype="bf16",
             pad=0, **LLAMA8B),
        # large trees, some beyond a word of the mask, seven heads a group of 64 columns, odd lengths, padding
        dict(name="tree_wide_f16", kind="tree_attn", q="64,117,33,1", kv="4001,6000,3277,900", words=2, page=128, dtype="f16", pad=9, Hq=28,
             Hkv=4, d=64),
        # one request with a draft model's distributions
        dict(name="verify_one", kind="verify", q="8", V=32000, dtype="f32", draft=True, most=8),
        # a full step of 64 requests over a large vocabulary
        dict(name="verify_many", kind="verify", q=_text([16] * 64), V=128000, dtype="f32", draft=True, most=16),
        # drafts that were looked up, not drawn: no distributions of their own; 16 bits, an odd vocabulary
        dict(name="verify_lookup_bf16", kind="verify", q=_text([4 + 3 * (i % 3) for i in range(24)]), V=50021, dtype="bf16", draft=False, most=6),
        # what 16 requests accepted, in all 32 layers
        dict(name="keep_layers", kind="keep", q=_text([16] * 16), kv=_text(_spread(16, 40, 90)), kept=_text([1 + i % 6 for i in range(16)]), layers=32,
             page=16, dtype="bf16", Hkv=8, d=128),
        # a cache thinned out: 20001 of 32768 tokens stay
        dict(name="keep_long", kind="keep", q="32768", kv="32768", kept="20001", layers=1, page=64, dtype="f16", Hkv=8, d=64),
        # after a step of 64 requests: a page here and there
        dict(name="trim_step", kind="trim", q=_text([16] * 64), kv=_text(_spread(64, 40, 16000)), kept=_text([1 + i % 7 for i in range(64)]), page=16),
        # 256 requests end at once
        dict(name="trim_release", kind="trim", q="", kv=_text(_spread(256, 300, 16000)), kept=_text([0] * 256), page=16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tree_map", "tree_attn", "tree_attn", "tree_attn", "verify", "verify", "keep", "trim"])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    if kind == "tree_map":
        B, most = _log_int(rng, 1, 256), _log_int(rng, 1, 200)
        q = [rng.randint(1, most) if rng.random() < 0.8 else 1 for _ in range(B)]
        q[0] = max(q[0], 9)
        return dict(kind=kind, q=_text(q), kv=_text(n + _log_int(rng, 1, 16384) for n in q), words=-(-max(q) // 64),
                    T=sum(q) + rng.choice([0, rng.randint(0, 64)]))
    if kind == "verify":
        V, dtype = _log_int(rng, 500, 128000), rng.choice(["f32", "f32", "bf16", "f16"])
        most = _log_int(rng, 2, 40)
        rows = min(1024 * 128000 // V, 2000)
        B = _log_int(rng, 1, max(1, min(128, rows // most)))
        return dict(kind=kind, q=_text(rng.randint(1, most) for _ in range(B)), V=V, dtype=dtype, draft=rng.random() < 0.7,
                    most=rng.choice([most, rng.randint(1, most)]))
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    dtype, d = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"]), rng.choice([64, 128, 128])
    if kind == "trim":
        B = _log_int(rng, 1, 512)
        if rng.random() < 0.5:
            q = [rng.randint(1, 64) for _ in range(B)]
            kv = [n + _log_int(rng, 1, 16384) for n in q]
            return dict(kind=kind, q=_text(q), kv=_text(kv), kept=_text(rng.randint(1, n) for n in q), page=page)
        kv = [_log_int(rng, 1, 16384) for _ in range(B)]
        return dict(kind=kind, q="", kv=_text(kv), kept=_text(rng.choice([0, rng.randint(0, n)]) for n in kv), page=page)
    if kind == "keep":
        shape = dict(page=page, dtype=dtype, Hkv=Hkv, d=d)
        if rng.random() < 0.7:
            B = _log_int(rng, 1, 48)
            q = [rng.randint(1, 64) for _ in range(B)]
            return dict(kind=kind, q=_text(q), kv=_text(n + rng.randint(0, 100) for n in q), kept=_text(rng.randint(1, min(n, 9)) for n in q),
                        layers=rng.choice([1, 4, rng.randint(1, 16)]), **shape)
        n = _log_int(rng, 100, 32768 // (2 if dtype == "f32" else 1))
        return dict(kind=kind, q=str(n), kv=str(n + rng.choice([0, rng.randint(0, 400)])), kept=str(rng.randint(1, n)), layers=1, **shape)
    B, most = _log_int(rng, 1, 48), rng.choice([_log_int(rng, 1, 64), _log_int(rng, 1, 64), _log_int(rng, 64, 300)])
    q = [rng.randint(1, most) for _ in range(B)]
    top = _log_int(rng, 64, 32768)
    kv = [n + rng.choice([0, rng.randint(max(1, top // 16), top), rng.randint(max(1, top // 16), top)]) for n in q]
    case = dict(kind=kind, words=-(-max(q) // 64) + rng.choice([0, 0, 1]), page=page, dtype=dtype, pad=rng.choice([0, 0, rng.randint(1, 40)]),
                Hq=Hkv * G, Hkv=Hkv, d=d)
    most_flops = 1.0e11 if dtype != "f32" else 1.0e10
    while True:
        case.update(q=_text(q), kv=_text(kv))
        w = work(case)
        if w["flops"] <= most_flops and w["bytes"] <= 1.1e9:
            return case
        big = max(range(len(q)), key=lambda i: kv[i])
        kv[big] = max(q[big], kv[big] * 2 // 3)
        if kv[big] == q[big]:
            if len(q) == 1:
                return case
            del q[big], kv[big]


# ----------------------------------------------------------------------------------------------- inputs
class _Gen:
    def __init__(self, seed):
        self.gpu = torch.Generator(device="cuda")
        self.gpu.manual_seed(seed * 7919 + 17)
        self.cpu = torch.Generator()
        self.cpu.manual_seed(seed * 104729 + 5)

    def act(self, L, H, d, dtype):
        """[L, H, d] activations with outlier channels."""
        s = torch.ones(H * d)
        s[torch.randperm(H * d, generator=self.cpu)[: max(1, round(0.01 * H * d))]] = 20.0
        s = s.view(1, H, d).to("cuda")
        out = torch.empty((L, H, d), dtype=dtype, device="cuda")
        for a in range(0, L, 1 << 16):
            out[a:a + (1 << 16)] = torch.randn((min(L - a, 1 << 16), H, d), generator=self.gpu, dtype=torch.float32, device="cuda").mul_(s)
        return out

    def ints(self, lo, hi, n):
        return torch.randint(lo, hi, (n,), generator=self.cpu).tolist()

    def parents(self, q):
        """A tree for each request: node 0 is its root, the others' parents are among the last few before, in order of depth."""
        out = []
        for n in q:
            tree = [-1]
            for r in self.ints(0, 1 << 30, n - 1):
                low = tree[-1] if len(tree) > 1 else 0
                tree.append(low + r % (min(len(tree) - low, 4)))
            out += tree
        return out

    def rows_of(self, q, kept):
        """Kept rows of each request: the first and others, in order."""
        out = torch.zeros((len(q), max(max(kept), 1)), dtype=torch.int32)
        for b, (n, k) in enumerate(zip(q, kept)):
            if k > 0:
                out[b, 0] = 0
                out[b, 1:k] = torch.sort(torch.randperm(n - 1, generator=self.cpu)[:k - 1])[0] + 1
        return out


def _dev32(values):
    return torch.tensor(values, dtype=torch.int32).to("cuda")


def _starts(q):
    start = [0]
    for n in q:
        start.append(start[-1] + n)
    return start


def _table(g, kv, P, spare):
    """(block table, number of pages, those of no request)"""
    need = [-(-n // P) for n in kv]
    ids = torch.randperm(sum(need) + spare, generator=g.cpu).to(torch.int32)
    table = torch.full((len(kv), max(need) + 1), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table.to("cuda"), sum(need) + spare, ids[at:]


def _prepare_verify(c, g):
    q, V, dt = _ints(c["q"]), c["V"], DTYPES[c["dtype"]]
    T, parents, start = sum(q), g.parents(q), _starts(q)
    owner = [b for b, n in enumerate(q) for _ in range(n)]
    up = torch.tensor([start[b] + max(p, 0) for b, p in zip(owner, parents)]).to("cuda")  # row of the parent
    target = torch.empty((T, V), dtype=dt, device="cuda")
    draft = torch.empty((T, V), dtype=dt, device="cuda") if c["draft"] else None
    tokens = torch.zeros(T, dtype=torch.int32, device="cuda")
    step = max(1, (1 << 26) // V)
    for a in range(0, T, step):
        logits = torch.randn((min(step, T - a), V), generator=g.gpu, device="cuda") * 2.5
        target[a:a + step] = torch.softmax(logits, -1)
        if draft is not None:
            draft[a:a + step] = torch.softmax(logits + 0.6 * torch.randn(logits.shape, generator=g.gpu, device="cuda"), -1)
    for a in range(0, T, step):
        if draft is not None:  # drawn from the parent's distribution
            x = draft[up[a:a + step]].float()
            tokens[a:a + step] = (x / torch.empty_like(x).exponential_(generator=g.gpu)).argmax(-1)
        else:  # likely ones: the most likely after some noise
            x = target[up[a:a + step]].float()
            tokens[a:a + step] = (x * torch.empty_like(x).uniform_(0.2, 1.0, generator=g.gpu)).argmax(-1)
    rand = lambda n: torch.rand(n, generator=g.gpu, dtype=torch.float64, device="cuda")  # noqa: E731
    B = len(q)
    new = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(case=c, target=target, draft=draft, tokens=tokens, parents=_dev32(parents), q_start=_dev32(start), u=rand(T), u_next=rand(B),
                kept=new(B, c["most"]), n_kept=new(B), next=new(B), most_rows=max(q))


def prepare(case, seed):
    g, c = _Gen(seed), case
    new = lambda n, dt=torch.int32: torch.zeros(n, dtype=dt, device="cuda")  # noqa: E731
    if c["kind"] == "verify":
        return _prepare_verify(c, g)
    kv = _ints(c["kv"])
    q = _ints(c["q"]) if c["q"] else []
    start = _starts(q)
    if c["kind"] == "tree_map":
        T = c["T"]
        return dict(case=c, parents=_dev32(g.parents(q) + [-1] * (T - sum(q))), q_start=_dev32(start), kv=_dev32(kv),
                    mask=new((T, c["words"]), torch.int64), positions=new(T), flags=new(len(kv)))
    P = c["page"]
    if c["kind"] == "trim":
        table, n_pages, spare = _table(g, kv, P, 40)
        free = torch.full((n_pages,), -1, dtype=torch.int32)
        free[:40] = spare
        return dict(case=c, kv=_dev32(kv), q_start=_dev32(start) if q else None, n_kept=_dev32(_ints(c["kept"])), table=table, free=free.to("cuda"),
                    count=_dev32([40]), lens=new(len(kv)), left=new(1), flags=new(1))
    dt, H, d = DTYPES[c["dtype"]], c["Hkv"], c["d"]
    table, n_pages, _ = _table(g, kv, P, 5)
    if c["kind"] == "keep":
        shape = (c["layers"], n_pages, H, P, d)
        K, V = (torch.randn(shape, generator=g.gpu, dtype=dt, device="cuda") for _ in range(2))
        kept = _ints(c["kept"])
        return dict(case=c, K=K, V=V, caches=[(K[i], V[i]) for i in range(c["layers"])], table=table, q_start=_dev32(start), kv=_dev32(kv),
                    kept=g.rows_of(q, kept).to("cuda"), n_kept=_dev32(kept))
    # a page's rows as they lie in the cache: [n_pages, H, P, d]
    Kp, Vp = (g.act(n_pages * P, H, d, dt).view(n_pages, P, H, d).transpose(1, 2).contiguous() for _ in range(2))
    T = sum(q) + c["pad"]
    up = g.parents(q)
    mask = torch.zeros((T, c["words"]), dtype=torch.int64)
    for b, n in enumerate(q):
        seen = []
        for i in range(n):
            p = up[start[b] + i]
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
            for w in range(c["words"]):
                bits = seen[i] >> 64 * w & (1 << 64) - 1
                mask[start[b] + i, w] = bits - (1 << 64) if bits >> 63 else bits
    return dict(case=c, Q=g.act(T, c["Hq"], d, dt).transpose(0, 1), Kp=Kp, Vp=Vp, table=table, q_start=_dev32(start), kv=_dev32(kv),
                mask=mask.to("cuda"), max_q=max(q), O=new((1, c["Hq"], T, d), torch.float32), lse=new((1, c["Hq"], T), torch.float32))


# ----------------------------------------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2605_25716_amd import binding as fb
    c = s["case"]
    if c["kind"] == "tree_map":
        fb.fedrag_tree_map(s["parents"], s["q_start"], s["kv"], c["words"], tree_mask=s["mask"], positions=s["positions"], flags=s["flags"])
        return {k: s[k] for k in ("mask", "positions", "flags")}
    if c["kind"] == "tree_attn":
        O, lse = fb.fedrag_paged_tree_attn(s["Q"], s["Kp"], s["Vp"], s["table"], s["q_start"], s["kv"], s["mask"], s["max_q"], O_part=s["O"],
                                           lse=s["lse"])
        return dict(O=O, lse=lse)
    if c["kind"] == "verify":
        fb.fedrag_tree_verify(s["target"], s["tokens"], s["parents"], s["q_start"], s["u"], s["u_next"], draft=s["draft"], kept=s["kept"],
                              n_kept=s["n_kept"], next_token=s["next"])
        return {k: s[k] for k in ("kept", "n_kept", "next")}
    if c["kind"] == "keep":
        fb.fedrag_paged_keep(s["caches"], s["table"], s["q_start"], s["kv"], s["kept"], s["n_kept"])
        return dict(K=s["K"], V=s["V"])
    fb.fedrag_paged_trim(s["kv"], s["n_kept"], s["table"], s["free"], s["count"], c["page"], q_start=s["q_start"], lens_out=s["lens"],
                         free_left=s["left"], flags=s["flags"])
    return {k: s[k] for k in ("lens", "free", "left", "flags")}


def _run_plain(s):
    return {"tree_map": _plain_map, "tree_attn": _plain_attn, "verify": _plain_verify, "keep": _plain_keep, "trim": _plain_trim}[s["case"]["kind"]](s)


def _plain_map(s):
    c = s["case"]
    T, N = c["T"], 64 * c["words"]
    start, kv = s["q_start"].long(), s["kv"].long()
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(start[1:], t, right=True)
    real = b < kv.numel()
    b = b.clamp(max=kv.numel() - 1)
    node = t - start[b]
    up = s["parents"].long()
    above = torch.where(real & (up >= 0), start[b] + up, T)  # row of the parent; T: there is none
    above = torch.cat([above, above.new_full((1,), T)])
    seen = torch.zeros((T + 1, N), dtype=torch.bool, device="cuda")
    seen[:T] = (node[:, None] == torch.arange(N, device="cuda")) & real[:, None]
    depth = torch.cat([(above[:T] < T).long(), above.new_zeros(1)])
    for _ in range(max(1, (N - 1).bit_length())):  # twice as many ancestors each time
        seen = seen | seen[above]
        depth = depth + depth[above]
        above = above[above]
    bits = torch.ones(64, dtype=torch.int64, device="cuda") << torch.arange(64, device="cuda")
    s["mask"].copy_((seen[:T].view(T, -1, 64).long() * bits).sum(-1))
    rows = start[1:] - start[:-1]
    s["positions"].copy_(torch.where(real, (kv - rows)[b] + depth[:T], -1))
    s["flags"].zero_()
    return {k: s[k] for k in ("mask", "positions", "flags")}


def _plain_attn(s):
    c = s["case"]
    q, kv, P, H, Hq, d = _ints(c["q"]), _ints(c["kv"]), c["page"], c["Hkv"], c["Hq"], c["d"]
    G, scale = Hq // H, d ** -0.5
    t0 = 0
    for b, (n, L) in enumerate(zip(q, kv)):
        ids = s["table"][b, :-(-L // P)].long()
        K = s["Kp"][ids].transpose(0, 1).reshape(H, -1, d)[:, :L].float()
        V = s["Vp"][ids].transpose(0, 1).reshape(H, -1, d)[:, :L].float()
        x = s["Q"][:, t0:t0 + n].reshape(H, G * n, d).float()
        S = torch.bmm(x, K.transpose(1, 2).contiguous()).view(H, G, n, L) * scale
        bit = torch.arange(n, device="cuda")
        seen = s["mask"][t0:t0 + n][:, bit // 64] >> (bit % 64) & 1
        S[..., L - n:] = torch.where(seen.bool(), S[..., L - n:], -math.inf)
        m = S.amax(-1, keepdim=True)
        S = torch.exp(S - m)
        total = S.sum(-1, keepdim=True)
        s["O"][0, :, t0:t0 + n] = (torch.bmm(S.view(H, G * n, L), V).view(H, G, n, d) / total).view(Hq, n, d)
        s["lse"][0, :, t0:t0 + n] = (m + torch.log(total)).view(Hq, n)
        t0 += n
    return dict(O=s["O"], lse=s["lse"])


def _whole(x):
    return torch.round(x * UNIT).long()


def _plain_verify(s):
    """All requests side by side: candidates come in order of their index, as a node's children and a child's own do."""
    c = s["case"]
    most, start = c["most"], s["q_start"].long()
    B, rows = start.numel() - 1, start[1:] - start[:-1]
    tokens, parents, u = s["tokens"].long(), s["parents"].long(), s["u"]
    at = torch.zeros(B, dtype=torch.int64, device="cuda")  # the node that each request is at
    n_kept = torch.ones_like(at)
    used = torch.zeros(B, dtype=torch.float64, device="cuda")  # C
    mass = torch.full_like(used, UNIT)                         # M, in units
    s["kept"].zero_()
    gone = torch.zeros((B, s["most_rows"]), dtype=torch.int64, device="cuda") - 1  # draft is None: tokens rejected at this node
    for i in range(1, s["most_rows"]):
        row = (start[:-1] + i).clamp(max=tokens.numel() - 1)
        asked = (i < rows) & (parents[row] == at) & (n_kept < most)
        x, here = tokens[row], start[:-1] + at
        p = s["target"][here, x].double()
        if s["draft"] is not None:
            q = s["draft"][here, x].double()
            left = (p - used / UNIT * q).clamp(min=0.0)
            yes = asked & (u[row] * q * mass < left * UNIT)
        else:
            left = torch.where((gone == x[:, None]).any(1), 0.0, p)
            yes = asked & (u[row] * mass < left * UNIT)
        no = asked & ~yes
        if s["draft"] is not None:
            used = torch.where(no, used + mass, used)
            which = no.nonzero()[:, 0]
            if which.numel():
                r = s["target"][here[which]].double() - (used[which] / UNIT)[:, None] * s["draft"][here[which]].double()
                mass[which] = _whole(r.clamp(min=0.0)).sum(-1).double()
        else:
            mass = torch.where(no, (mass - _whole(left)).clamp(min=0.0), mass)
            gone[:, i] = torch.where(no, x, gone[:, i])
        s["kept"].scatter_(1, n_kept.clamp(max=most - 1)[:, None],
                           torch.where(yes, i, s["kept"].gather(1, n_kept.clamp(max=most - 1)[:, None])[:, 0])[:, None].int())
        at = torch.where(yes, i, at)
        n_kept = n_kept + yes.long()
        used = torch.where(yes, 0.0, used)
        mass = torch.where(yes, UNIT, mass)
        gone = torch.where(yes[:, None], -1, gone)
    here = start[:-1] + at
    p = s["target"][here].double()
    weight = _whole(p)
    if s["draft"] is not None:
        left = _whole((p - (used / UNIT)[:, None] * s["draft"][here].double()).clamp(min=0.0))
    else:
        left = torch.cat([weight, weight.new_zeros((B, 1))], 1).scatter_(1, torch.where(gone < 0, weight.shape[1], gone), 0)[:, :-1]
    weight = torch.where(left.sum(-1, keepdim=True) > 0, left, weight)
    total = weight.sum(-1)
    threshold = torch.minimum(torch.floor(s["u_next"] * total.double()).long(), total - 1)
    s["next"].copy_((torch.cumsum(weight, -1) > threshold[:, None]).int().argmax(-1))
    s["n_kept"].copy_(n_kept)
    return {k: s[k] for k in ("kept", "n_kept", "next")}


def _plain_keep(s):
    c = s["case"]
    P, start = c["page"], s["q_start"].long()
    base = s["kv"].long() - (start[1:] - start[:-1])
    j = torch.arange(s["kept"].shape[1], device="cuda")
    b, j = (j[None, :] < s["n_kept"][:, None]).nonzero(as_tuple=True)
    source, to = base[b] + s["kept"].long()[b, j], base[b] + j
    table = s["table"].long()
    from_page, to_page = table[b, source // P], table[b, to // P]
    for pages in (s["K"], s["V"]):
        pages[:, to_page, :, to % P] = pages[:, from_page, :, source % P]
    return dict(K=s["K"], V=s["V"])


def _plain_trim(s):
    P, table = s["case"]["page"], s["table"]
    kv, lens = s["kv"].long(), s["n_kept"].long()
    if s["q_start"] is not None:
        lens = kv - (s["q_start"][1:] - s["q_start"][:-1]) + lens
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    freed = (col >= ((lens + P - 1) // P)[:, None]) & (col < ((kv + P - 1) // P)[:, None])
    ids = table[freed]
    top = s["count"].long()
    s["free"][top + torch.arange(ids.numel(), device="cuda")] = ids
    s["lens"].copy_(lens)
    s["left"].copy_(top + ids.numel())
    s["flags"].zero_()
    return {k: s[k] for k in ("lens", "free", "left", "flags")}


# ----------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    if case["kind"] != "tree_attn":  # whole numbers and copies
        return None
    s, c = prepare(case, seed), case
    q, kv, P, Hq = _ints(c["q"]), _ints(c["kv"]), c["page"], c["Hq"]
    group = Hq // c["Hkv"]
    masks = s["mask"].cpu().tolist()
    O = torch.zeros(s["O"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    begin = 0
    for b, n in enumerate(q):
        hidden = torch.zeros((n, kv[b]), dtype=torch.bool)
        for i in range(n):
            for node in range(n):
                hidden[i, kv[b] - n + node] = not (masks[begin + i][node // 64] >> node % 64) & 1
        hidden = hidden.to("cuda")
        key = torch.arange(kv[b], device="cuda")
        page, at = s["table"][b].long()[key // P], key % P
        rows = slice(begin, begin + n)
        for h in range(Hq):
            K, V = s["Kp"][page, h // group, at].double(), s["Vp"][page, h // group, at].double()
            logit = (torch.matmul(s["Q"][h, rows].double(), K.t().contiguous()) / math.sqrt(c["d"])).masked_fill(hidden, -math.inf)
            norm = torch.logsumexp(logit, -1)
            O[0, h, rows] = torch.matmul(torch.exp(logit - norm[:, None]), V)
            lse[0, h, rows] = norm
        begin += n
    return dict(O=O, lse=lse)


# ----------------------------------------------------------------------------------------------- what it cannot do without
def work(case):
    c = case
    q = _ints(c["q"]) if c["q"] else []
    if c["kind"] == "tree_map":
        return {"bytes": 8 * len(q) + 4 * sum(q) + (4 + 8 * c["words"]) * c["T"], "flops": 0}
    if c["kind"] == "verify":  # a request's tree, and the row or two of its last node
        size = DTYPES[c["dtype"]].itemsize
        return {"bytes": len(q) * (1 + c["draft"]) * c["V"] * size + 16 * sum(q) + 20 * len(q), "flops": 2 * len(q) * c["V"]}
    kv = _ints(c["kv"])
    if c["kind"] == "trim":
        kept = _ints(c["kept"])
        lens = [L - n + k for L, n, k in zip(kv, q, kept)] if q else kept
        return {"bytes": 16 * len(kv) + 8 * sum(-(-a // c["page"]) - -(-b // c["page"]) for a, b in zip(kv, lens)) + 12, "flops": 0}
    size, d = DTYPES[c["dtype"]].itemsize, c["d"]
    if c["kind"] == "keep":
        kept = _ints(c["kept"])  # (the first row stays where it is)
        return {"bytes": 4 * c["layers"] * sum(max(k - 1, 0) for k in kept) * c["Hkv"] * d * size + 4 * sum(kept) + 16 * len(q), "flops": 0}
    pairs = sum(n * (L - n) + n * max(1, n.bit_length()) for n, L in zip(q, kv))  # (what a row sees of its tree is about its depth)
    read = 2 * sum(kv) * c["Hkv"] * d * size + sum(q) * (c["Hq"] * d * size + 8 * c["words"])
    return {"bytes": read + sum(q) * c["Hq"] * (d + 1) * 4 + 4 * sum(-(-L // c["page"]) for L in kv), "flops": 4 * d * c["Hq"] * pairs}
