"""The paged cache of a serving node and the attention that reads it: the work whose speed counts.

Kinds of cases (key "kind"):
  map    block tables, row offsets, slots and positions of one step, from the requests' lengths.
  write  the step's new K, V rows (strided views of a projection's output, or dense per head) into the cache's pages.
  attn   attention of the step's rows over the pages: a decoded token per request, a chunk of a prompt, or both at once.

"q" and "kv" are the requests' new rows and their keys (the new rows among them), comma separated.  Causal attention is
the Inquirer's own part over its plaintext cache: activations N(0,1) with 1 % of the (head, channel) axis scaled by 20.
Attention without a mask is a Compute Node's over scrambled rows: those activations times an orthogonal matrix per KV head.
Pages are handed out in random order, as after a while of serving.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LLAMA8B = dict(Hq=32, Hkv=8, d=128)


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _spread(n, lo, hi):
    """n lengths from hi down to lo, evenly over their logarithm, none of them round."""
    if n == 1:
        return [hi]
    return [max(1, int(round(hi * (lo / hi) ** (i / (n - 1)))) - (i % 3)) for i in range(n)]


def listed():
    ragged = _spread(64, 1000, 32768)
    mixed = _spread(24, 300, 8192)
    return [
        # one decoded token of four requests: what a step's bookkeeping costs at the least
        dict(name="map_token", kind="map", q="1,1,1,1", kv="193,4097,801,32", page=16, T=4),
        # a step of 256 requests, most of them at one token, a few with a chunk of their prompt; rows padded to a round number
        dict(name="map_step", kind="map", q=_text([1] * 250 + [512, 777, 64, 1024, 1, 333]),
             kv=_text(_spread(250, 40, 16000) + [512, 4001, 64, 9000, 1, 3277]), page=32, T=3008),
        # admission of a large batch of prompts at once
        dict(name="map_prompts", kind="map", q=_text([4096 - 13 * (i % 17) for i in range(32)]),
             kv=_text([4096 - 13 * (i % 17) + (1000 if i % 4 == 0 else 0) for i in range(32)]), page=16, T=131072),
        # the rows of one decoded token
        dict(name="write_token", kind="write", T=1, Hkv=8, d=128, dtype="bf16", page=16, n_pages=4096, fused=4, live=1),
        # a prompt of odd length out of a fused projection, 64 columns in fp16
        dict(name="write_chunk_f16", kind="write", T=4001, Hkv=8, d=64, dtype="f16", page=64, n_pages=512, fused=4, live=3990),
        # a whole context of scrambled rows, dense per head as Enc leaves them
        dict(name="write_context", kind="write", T=32768, Hkv=8, d=128, dtype="bf16", page=128, n_pages=300, fused=0, live=32768),
        # one decoded token of one short request, as the paper's Short workload has it: latency
        dict(name="token_192", kind="attn", q="1", kv="192", causal=True, page=16, dtype="bf16", pad=0, **LLAMA8B),
        # a decoding step of 64 requests of very unequal lengths
        dict(name="decode_ragged", kind="attn", q=_text([1] * 64), kv=_text(ragged), causal=True, page=16, dtype="bf16", pad=0,
             **LLAMA8B),
        # a chunk of a long prompt over what is in the cache already
        dict(name="chunk_16k", kind="attn", q="1024", kv="16384", causal=True, page=64, dtype="bf16", pad=0, **LLAMA8B),
        # decoding requests and the chunks of three prompts in one step, rows padded behind the last
        dict(name="mixed_step", kind="attn", q=_text([1] * 24 + [512, 777, 2048]), kv=_text(mixed + [512, 4001, 2048]), causal=True,
             page=32, dtype="bf16", pad=63, **LLAMA8B),
        # a Compute Node's contexts of odd lengths for the queries of three requests, fp16, 64 columns, seven heads a group
        dict(name="remote_f16", kind="attn", q="117,1,64", kv="4001,3277,6000", causal=False, page=128, dtype="f16", pad=0, Hq=28,
             Hkv=4, d=64),
        # the fp32 path of a parity run: odd chunks, one of them a token
        dict(name="parity_f32", kind="attn", q="33,1,70", kv="500,1025,70", causal=True, page=16, dtype="f32", pad=2, Hq=8, Hkv=2,
             d=128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["map", "write", "attn", "attn", "attn", "attn"])
    if kind == "map":
        B, page = _log_int(rng, 1, 512), rng.choice([16, 32, 64, 128, 256])
        top = _log_int(rng, 1, 131072 // B)
        q = [1 if rng.random() < 0.5 else rng.randint(0, top) for _ in range(B)]
        q[0] = max(1, q[0])
        return dict(kind=kind, q=_text(q), kv=_text(n + rng.choice([0, 0, _log_int(rng, 1, 16384)]) for n in q), page=page,
                    T=sum(q) + rng.choice([0, rng.randint(0, 64)]))
    if kind == "write":
        T, Hkv, d = _log_int(rng, 1, 32768), rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
        page, dtype = rng.choice([16, 32, 64, 128, 256]), rng.choice(["bf16", "bf16", "f16", "f32"])
        if dtype == "f32":
            T = max(1, T // 2)
        return dict(kind=kind, T=T, Hkv=Hkv, d=d, dtype=dtype, page=page, n_pages=-(-T // page) + rng.randint(1, 256),
                    fused=rng.choice([0, 1, 4]), live=max(1, T - rng.choice([0, 0, rng.randint(0, 9)])))
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    shape = dict(Hq=Hkv * G, Hkv=Hkv, d=rng.choice([64, 128, 128]), page=rng.choice([16, 16, 32, 64, 128, 256]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
    form = rng.choice(["decode", "decode", "chunk", "mixed"])
    if form == "decode":
        B = _log_int(rng, 1, 96)
        q = [1] * B
        top = _log_int(rng, 64, 32768)
        kv = [rng.randint(max(1, top // 16), top) for _ in range(B)]
    else:
        n = rng.choice([1, 1, 2, 3])
        q = [_log_int(rng, 2, 2048) for _ in range(n)]
        kv = [m + rng.choice([0, _log_int(rng, 16, 16384)]) for m in q]
        if form == "mixed":
            for _ in range(_log_int(rng, 1, 32)):
                q.append(1)
                kv.append(_log_int(rng, 16, 8192))
    case = dict(kind=kind, causal=rng.random() < 0.75, dtype=dtype, pad=rng.choice([0, 0, rng.randint(1, 40)]), **shape)
    most = 2.0e11 if dtype != "f32" else 1.0e10
    while True:
        case.update(q=_text(q), kv=_text(kv))
        w = work(case)
        if w["flops"] <= most and w["bytes"] <= 2.2e9:
            return case
        big = max(range(len(q)), key=lambda i: q[i] * kv[i])
        if q[big] > 64:
            q[big] = q[big] * 2 // 3
        kv[big] = max(q[big], kv[big] * 2 // 3)
        if kv[big] == q[big] == 1:
            return case


# ----------------------------------------------------------------------------------------------- inputs
def _ints(text):
    return [int(x) for x in text.split(",")]


class _Gen:
    def __init__(self, seed):
        self.gpu = torch.Generator(device="cuda")
        self.gpu.manual_seed(seed * 7919 + 17)
        self.cpu = torch.Generator()
        self.cpu.manual_seed(seed * 104729 + 5)

    def act(self, L, H, d, dtype, mix):
        """[L, H, d] activations with outlier channels; mix: times one orthogonal matrix per head, as after Enc."""
        s = torch.ones(H * d)
        s[torch.randperm(H * d, generator=self.cpu)[: max(1, round(0.01 * H * d))]] = 20.0
        s = s.view(1, H, d).to("cuda")
        phi = None
        if mix is not None:
            phi = mix.repeat_interleave(H // mix.shape[0], 0).to("cuda").float()
        out = torch.empty((L, H, d), dtype=dtype, device="cuda")
        for a in range(0, L, 1 << 16):
            x = torch.randn((min(L - a, 1 << 16), H, d), generator=self.gpu, dtype=torch.float32, device="cuda").mul_(s)
            out[a:a + x.shape[0]] = x if phi is None else torch.bmm(x.transpose(0, 1).contiguous(), phi).transpose(0, 1)
        return out

    def haar(self, H, d):
        q, r = torch.linalg.qr(torch.randn((H, d, d), generator=self.cpu, dtype=torch.float64))
        return q * torch.sign(torch.diagonal(r, dim1=-2, dim2=-1)).unsqueeze(-2)

    def perm(self, n):
        return torch.randperm(n, generator=self.cpu)


def _dev32(values):
    return torch.tensor(values, dtype=torch.int32).to("cuda")


def prepare(case, seed):
    g, c = _Gen(seed), case
    if c["kind"] == "map":
        q, kv, P = _ints(c["q"]), _ints(c["kv"]), c["page"]
        cached = [b - a for a, b in zip(q, kv)]
        had, need = [-(-n // P) for n in cached], [-(-n // P) for n in kv]
        columns = max(need) + 3
        ids = g.perm(sum(need) + 40).to(torch.int32)
        table = torch.full((len(q), columns), -1, dtype=torch.int32)
        at = 0
        for b, h in enumerate(had):
            table[b, :h] = ids[at:at + h]
            at += h
        free = ids[at:].contiguous()
        B, T = len(q), c["T"]
        new = lambda n, dt: torch.zeros(n, dtype=dt, device="cuda")  # noqa: E731
        return dict(case=c, cached=_dev32(cached), new=_dev32(q), free=free.to("cuda"), count=_dev32([free.numel()]),
                    table=table.to("cuda"), q_start=new(B + 1, torch.int32), kv=new(B, torch.int32), slots=new(T, torch.int64),
                    positions=new(T, torch.int32), left=new(1, torch.int32), flags=new(1, torch.int32))
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "write":
        T, H, d, P, n = c["T"], c["Hkv"], c["d"], c["page"], c["n_pages"]
        if c["fused"]:  # [T, (query heads, K, V)] of one projection; K and V are views of it
            x = g.act(T, (c["fused"] + 2) * H, d, dt, None)
            K, V = x[:, c["fused"] * H:(c["fused"] + 1) * H].transpose(0, 1), x[:, (c["fused"] + 1) * H:].transpose(0, 1)
        else:           # [H, T, d] as Enc leaves it
            mix = g.haar(H, d)
            K, V = (g.act(T, H, d, dt, mix).transpose(0, 1).contiguous() for _ in range(2))
        base = -(-T // P)
        pages = g.perm(n)[:base]
        first = int(torch.randint(0, P, (1,), generator=g.cpu)) if base * P - T > 0 else 0
        first = min(first, base * P - T)
        t = torch.arange(T) + first
        slots = pages[t // P] * P + t % P
        slots[c["live"]:] = -1
        return dict(case=c, K=K, V=V, slots=slots.to("cuda"), Kp=torch.zeros((n, H, P, d), dtype=dt, device="cuda"),
                    Vp=torch.zeros((n, H, P, d), dtype=dt, device="cuda"))
    q, kv, P, H, Hq, d = _ints(c["q"]), _ints(c["kv"]), c["page"], c["Hkv"], c["Hq"], c["d"]
    need = [-(-n // P) for n in kv]
    n_pages = sum(need) + 5
    mix = None if c["causal"] else g.haar(H, d)
    ids = g.perm(n_pages).to(torch.int32)
    table = torch.full((len(q), max(need) + 1), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    T = sum(q) + c["pad"]
    # a page's rows as they lie in the cache: [n_pages, H, P, d]
    Kp, Vp = (g.act(n_pages * P, H, d, dt, mix).view(n_pages, P, H, d).transpose(1, 2).contiguous() for _ in range(2))
    start = [0]
    for n in q:
        start.append(start[-1] + n)
    # queries: a projection's output [T, Hq, d], or dense per head as Enc leaves them
    Q = g.act(T, Hq, d, dt, mix).transpose(0, 1)
    if not c["causal"]:
        Q = Q.contiguous()
    return dict(case=c, Q=Q, Kp=Kp, Vp=Vp, table=table.to("cuda"), q_start=_dev32(start), kv=_dev32(kv), max_q=max(q),
                O=torch.zeros((1, Hq, T, d), dtype=torch.float32, device="cuda"),
                lse=torch.zeros((1, Hq, T), dtype=torch.float32, device="cuda"))


# ----------------------------------------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2605_25716_amd import binding as fb
    c = s["case"]
    if c["kind"] == "map":
        fb.fedrag_paged_map(s["cached"], s["new"], s["table"], s["free"], s["count"], c["page"], c["T"], q_start=s["q_start"],
                            kv_lens=s["kv"], slots=s["slots"], positions=s["positions"], free_left=s["left"], flags=s["flags"])
        return _map_out(s)
    if c["kind"] == "write":
        fb.fedrag_paged_write(s["K"], s["V"], s["slots"], s["Kp"], s["Vp"])
        return dict(K=s["Kp"], V=s["Vp"])
    O, lse = fb.fedrag_paged_attn(s["Q"], s["Kp"], s["Vp"], s["table"], s["q_start"], s["kv"], s["max_q"], causal=c["causal"],
                                  O_part=s["O"], lse=s["lse"])
    return dict(O=O, lse=lse)


def _map_out(s):
    return {k: s[k] for k in ("table", "q_start", "kv", "slots", "positions", "left", "flags")}


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "map":
        return _plain_map(s)
    if c["kind"] == "write":
        P, slots = c["page"], s["slots"]
        live = slots >= 0
        page, at = slots[live] // P, slots[live] % P
        for rows, pages in ((s["K"], s["Kp"]), (s["V"], s["Vp"])):
            pages[page, :, at] = rows.transpose(0, 1)[live]
        return dict(K=s["Kp"], V=s["Vp"])
    return _plain_attn(s)


def _plain_map(s):
    c = s["case"]
    P, T = c["page"], c["T"]
    cached, new, table = s["cached"].long(), s["new"].long(), s["table"]
    B, columns = table.shape
    end = torch.cumsum(new, 0)
    s["q_start"][0] = 0
    s["q_start"][1:] = end
    kv = cached + new
    s["kv"].copy_(kv)
    had = (cached + P - 1) // P
    want = (kv + P - 1) // P - had
    page_end = torch.cumsum(want, 0)
    col = torch.arange(columns, device="cuda")[None, :]
    fresh = (col >= had[:, None]) & (col < (had + want)[:, None])
    nth = (page_end - want)[:, None] + col - had[:, None]
    top = s["count"].long()
    ids = s["free"].long()[torch.clamp(top - 1 - nth, 0, s["free"].numel() - 1)]
    table.copy_(torch.where(fresh, ids, table.long()))
    s["left"].copy_(top - page_end[-1:])
    s["flags"].zero_()
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(end, t, right=True)
    real = b < B
    b = torch.clamp(b, max=B - 1)
    pos = cached[b] + t - (end - new)[b]
    slot = table.long()[b, torch.clamp(pos // P, 0, columns - 1)] * P + pos % P
    s["slots"].copy_(torch.where(real, slot, -1))
    s["positions"].copy_(torch.where(real, pos, -1))
    return _map_out(s)


def _plain_attn(s):
    c = s["case"]
    q, kv, P, H, Hq, d = _ints(c["q"]), _ints(c["kv"]), c["page"], c["Hkv"], c["Hq"], c["d"]
    G, scale = Hq // H, d ** -0.5
    t0 = 0
    for b, (n, L) in enumerate(zip(q, kv)):
        if n == 0:
            continue
        ids = s["table"][b, :-(-L // P)].long()
        K = s["Kp"][ids].transpose(0, 1).reshape(H, -1, d)[:, :L].float()
        V = s["Vp"][ids].transpose(0, 1).reshape(H, -1, d)[:, :L].float()
        Kt = K.transpose(1, 2).contiguous()
        for a in range(0, n, 1024):
            e = min(n, a + 1024)
            x = s["Q"][:, t0 + a:t0 + e].reshape(H, G * (e - a), d).float()
            S = torch.bmm(x, Kt) * scale
            if c["causal"]:
                seen = torch.arange(L, device="cuda")[None, :] <= torch.arange(a, e, device="cuda")[:, None] + (L - n)
                S = torch.where(seen.repeat(G, 1)[None], S, -math.inf)
            m = S.amax(-1, keepdim=True)
            S = torch.exp(S - m)
            total = S.sum(-1, keepdim=True)
            s["O"][0, :, t0 + a:t0 + e] = (torch.bmm(S, V) / total).view(Hq, e - a, d)
            s["lse"][0, :, t0 + a:t0 + e] = (m + torch.log(total)).view(Hq, e - a)
        t0 += n
    return dict(O=s["O"], lse=s["lse"])


# ----------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    if case["kind"] != "attn":  # whole numbers and copies
        return None
    s, c = prepare(case, seed), case
    q, kv, P, Hq = _ints(c["q"]), _ints(c["kv"]), c["page"], c["Hq"]
    group = Hq // c["Hkv"]
    O = torch.zeros(s["O"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    begin = 0
    for b in range(len(q)):
        rows = torch.arange(begin, begin + q[b], device="cuda")
        begin += q[b]
        key = torch.arange(kv[b], device="cuda")
        page, at = s["table"][b].long()[key // P], key % P
        for h in range(Hq):
            K, V = s["Kp"][page, h // group, at].double(), s["Vp"][page, h // group, at].double()
            for part in rows.split(2048):
                logit = torch.matmul(s["Q"][h, part].double(), K.t().contiguous()) / math.sqrt(c["d"])
                if c["causal"]:
                    own_place = kv[b] - q[b] + (part - rows[0])
                    logit = logit.masked_fill(key[None, :] > own_place[:, None], -math.inf)
                norm = torch.logsumexp(logit, -1)
                O[0, h, part] = torch.matmul(torch.exp(logit - norm[:, None]), V)
                lse[0, h, part] = norm
    return dict(O=O, lse=lse)


# ----------------------------------------------------------------------------------------------- what it cannot do without
def work(case):
    c = case
    if c["kind"] == "map":
        q, kv, P = _ints(c["q"]), _ints(c["kv"]), c["page"]
        fresh = sum(-(-b // P) - -(-(b - a) // P) for a, b in zip(q, kv))
        return {"bytes": 16 * len(q) + 8 * fresh + 12 * c["T"] + 16, "flops": 0}
    size = DTYPES[c["dtype"]].itemsize
    if c["kind"] == "write":
        return {"bytes": 4 * c["live"] * c["Hkv"] * c["d"] * size + 8 * c["T"], "flops": 0}
    q, kv, d = _ints(c["q"]), _ints(c["kv"]), c["d"]
    pairs = sum(n * L - (n * (n - 1) // 2 if c["causal"] else 0) for n, L in zip(q, kv))
    read = 2 * sum(L for n, L in zip(q, kv) if n) * c["Hkv"] * d * size + sum(q) * c["Hq"] * d * size
    return {"bytes": read + sum(q) * c["Hq"] * (d + 1) * 4 + 4 * sum(-(-L // c["page"]) for L in kv),
            "flops": 4 * d * c["Hq"] * pairs}
