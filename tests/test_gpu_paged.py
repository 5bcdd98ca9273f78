"""The paged cache on the GPU: planning a step, writing its rows, attending to them; each against its plain statement."""
import numpy as np
import pytest
import torch

import paged_ref as R
from paper_2605_25716_amd import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FILL = 7.0


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int64).astype(np.int32)).to(DEV)


# ----------------------------------------------------------------------------------------------- map
def _map_case(B, seed, page, columns, top, zero_new=0.2, T_more=3, stack=None):
    rng = np.random.default_rng(seed)
    cached = rng.integers(0, top, B)
    new = rng.integers(1, top, B) * (rng.random(B) >= zero_new)
    table = np.full((B, columns), -7, np.int64)
    for b in range(B):
        table[b, :min(columns, -(-cached[b] // page))] = rng.integers(0, 10 ** 6, min(columns, -(-cached[b] // page)))
    need = int(sum(-(-(c + n) // page) - -(-c // page) for c, n in zip(cached, new)))
    free = rng.permutation(need + 9) + 10 ** 6
    return cached, new, table, free, (need + 4 if stack is None else stack), page, int(new.sum()) + T_more


def _run_map(cached, new, table, free, count, page, T, in_place=False):
    c, n, tb, fr, fc = i32(cached), i32(new), i32(table), i32(free), i32([count])
    kw = dict(kv_lens=c, free_left=fc) if in_place else {}
    got = fb.fedrag_paged_map(c, n, tb, fr, fc, page, T, **kw)
    return got, tb, c, fc


def _check_map(got, table, ref):
    q_start, kv, slots, pos, left, flags = (x.cpu().numpy() for x in got)
    r = dict(zip(("q_start", "kv", "table", "slots", "positions", "left", "flags"), ref))
    np.testing.assert_array_equal(q_start, r["q_start"])
    np.testing.assert_array_equal(kv, r["kv"])
    np.testing.assert_array_equal(table.cpu().numpy(), r["table"])
    np.testing.assert_array_equal(slots, r["slots"])
    np.testing.assert_array_equal(pos, r["positions"])
    assert int(left[0]) == r["left"] and int(flags[0]) == r["flags"]


@pytest.mark.parametrize("B,page,columns,top", [(1, 16, 4, 30), (2, 256, 3, 300), (63, 16, 9, 60), (64, 32, 40, 500), (65, 64, 9, 200),
                                                (1023, 16, 3, 9), (1024, 16, 3, 9), (1025, 128, 2, 9), (2300, 16, 2, 12), (9, 16, 400, 3000),
                                                (40, 16, 200, 1400)])
def test_map(B, page, columns, top):
    case = _map_case(B, B + page, page, columns, top)
    got, table, _, _ = _run_map(*case)
    _check_map(got, table, R.map_ref(*case))


@pytest.mark.parametrize("what", ["stack", "empty_stack", "columns", "rows", "negative", "no_rows", "count_above", "count_below", "holes", "huge"])
def test_map_out_of_the_ordinary(what):
    for B, page, columns, top, T_more in ((5, 16, 6, 50, 0), (300, 32, 70, 900, 5000)):  # one launch, and two
        cached, new, table, free, count, page, T = _map_case(B, 3, page, columns, top, T_more=T_more)
        if what == "stack":
            count = count // 2
        if what == "empty_stack":
            free, count = free[:0], 0
        if what == "columns":
            table = table[:, :columns // 3]
        if what == "rows":
            T = int(new.sum()) * 2 // 3
        if what == "negative":
            cached[B // 2], new[B // 3] = -5, -2 ** 31
        if what == "no_rows":
            T = 0
        if what == "count_above":
            count = len(free) + 1
        if what == "count_below":
            count = -1
        if what == "holes":
            table[:, 0] = -1
        if what == "huge":
            cached[B // 2], cached[B // 3], new[B - 1] = 2 ** 31 - 1, 2 ** 31 - 5, 2 ** 31 - 1
        got, tb, _, _ = _run_map(cached, new, table, free, count, page, T)
        _check_map(got, tb, R.map_ref(cached, new, table, free, count, page, T))


def test_map_of_no_requests():
    got = fb.fedrag_paged_map(i32([]), i32([]), torch.empty((0, 4), dtype=torch.int32, device=DEV), i32([3, 4]), i32([2]), 16, 5)
    q_start, kv, slots, pos, left, flags = (x.cpu().tolist() for x in got)
    assert q_start == [0] and kv == [] and slots == [-1] * 5 and pos == [-1] * 5 and left == [2] and flags == [0]


@pytest.mark.parametrize("B,T", [(3, 8), (300, 9000)])
def test_map_in_place_replayed(B, T):
    """kv_lens is cached_lens and free_left is free_count: every replay of a recorded step is the next one."""
    page, columns = 16, 40
    rng = np.random.default_rng(5)
    cached, new = rng.integers(0, 40, B), rng.integers(0, 2 if T < 100 else 30, B)
    table = np.full((B, columns), -1)
    free = rng.permutation(B * columns)
    at = 0
    for b in range(B):
        h = -(-int(cached[b]) // page)
        table[b, :h] = 10 ** 6 + np.arange(at, at + h)
        at += h
    c, n, tb, fr, fc = i32(cached), i32(new), i32(table), i32(free), i32([len(free)])
    out = {k: torch.zeros(s, dtype=d, device=DEV) for k, s, d in (("q_start", B + 1, torch.int32), ("slots", T, torch.int64),
                                                                  ("positions", T, torch.int32), ("flags", 1, torch.int32))}
    step = lambda: fb.fedrag_paged_map(c, n, tb, fr, fc, page, T, kv_lens=c, free_left=fc, **out)  # noqa: E731
    count = len(free)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(4):
        graph.replay() if k != 2 else step()  # an eager step between the replays
        torch.cuda.synchronize()
        ref = R.map_ref(cached, new, table, free, count, page, T)
        _check_map(got, tb, ref)
        cached, table, count = ref[1], ref[2], ref[5]


# ----------------------------------------------------------------------------------------------- write
def _bits(x):
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,H,d,page,form", [(1, 8, 128, 16, "fused"), (17, 1, 64, 16, "dense"), (300, 3, 128, 64, "tokens"),
                                             (33, 2, 64, 256, "fused"), (129, 5, 128, 32, "dense"), (70, 2, 64, 128, "one_row")])
def test_write(dt, T, H, d, page, form):
    rng = np.random.default_rng(T)
    n = -(-T // page) + 3
    g = torch.Generator().manual_seed(T)
    mk = lambda *s: torch.randn(s, generator=g).to(DT[dt])  # noqa: E731
    if form == "fused":
        x = mk(T, 4 * H, d)
        K, V = x[:, H:2 * H].transpose(0, 1), x[:, 3 * H:].transpose(0, 1)
    elif form == "tokens":
        K, V = mk(T, H, d).transpose(0, 1), mk(H, T, d)
    elif form == "one_row":  # one row for all tokens
        K, V = mk(H, 1, d).expand(H, T, d), mk(1, 1, d).expand(H, T, d)
    else:
        K, V = mk(1, H, T, d), mk(1, H, T, d)
    K.flatten()[:1].fill_(float("nan"))
    slots = torch.from_numpy(rng.permutation(n * page)[:T].astype(np.int64))
    for i, s in enumerate((-1, n * page, -2 ** 40, 2 ** 62, n * page + 5)):
        if T > 16:
            slots[3 * i] = s
    pages = torch.full((n, 2, H, page, d), FILL, dtype=DT[dt])  # K and V in turns
    dev = pages.to(DEV)
    # views of the same strides on the device (a copy of an expanded tensor would be dense)
    to = lambda x: x.to(DEV) if form != "one_row" else x[:, :1].to(DEV).expand(x.shape)  # noqa: E731
    if form == "one_row":
        V = mk(H, 1, d).expand(H, T, d)
    if form == "fused":
        xd = x.to(DEV)
        Kd, Vd = xd[:, H:2 * H].transpose(0, 1), xd[:, 3 * H:].transpose(0, 1)
    else:
        Kd, Vd = to(K), to(V)
    fb.fedrag_paged_write(Kd, Vd, slots.to(DEV), dev[:, 0], dev[:, 1])
    for i, rows in ((0, K), (1, V)):
        want = R.write_ref(rows.reshape(H, T, d), slots, pages[:, i])
        assert torch.equal(_bits(dev[:, i].cpu()), _bits(want))


def test_write_far_slots():
    """A cache whose byte offsets pass 32 bits (and its element offsets, 31)."""
    H, d, page, n = 1, 64, 256, 150000
    K, V = (torch.randn((H, 3, d), device=DEV).to(torch.bfloat16) for _ in range(2))
    Kp, Vp = (torch.zeros((n, H, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    slots = torch.tensor([n * page - 1, 0, 2 ** 25 + 3], device=DEV)
    fb.fedrag_paged_write(K, V, slots, Kp, Vp)
    for rows, pages in ((K, Kp), (V, Vp)):
        flat = pages.view(n * page, d)
        assert torch.equal(flat[slots], rows[0]) and int((flat != 0).any(1).sum()) == 3
    # and attention that reads them there: the last page, the first and one in the middle as one request's tokens
    table = i32([[n - 1, 0, 2 ** 25 // page]])
    Q = torch.randn((2, 1, d), device=DEV).to(torch.bfloat16)
    O, lse = fb.fedrag_paged_attn(Q, Kp, Vp, table, i32([0, 1]), i32([3 * page]), 1, causal=False)
    keep = torch.tensor([n - 1, 0, 2 ** 25 // page], device=DEV)
    ref = R.attn_ref(Q.cpu(), Kp[keep].cpu(), Vp[keep].cpu(), [[0, 1, 2]], [0, 1], [3 * page], False, d ** -0.5)
    R.check_attn(O, lse, ref, FILL, "far")


# ----------------------------------------------------------------------------------------------- attention
def _attn_case(q, kv, Hq, Hkv, d, page, dt, seed=0, pad=0, more_columns=1, outliers=False):
    g = torch.Generator().manual_seed(int(seed * 1009 + sum(q) + 7 * sum(kv) + d))
    need = [-(-max(n, 0) // page) for n in kv]
    n_pages = sum(need) + 2
    ids = torch.randperm(n_pages, generator=g).numpy()
    table = np.full((len(q), max(need + [0]) + more_columns), -1, np.int64)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    mk = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    Q, Kp, Vp = mk(Hq, sum(q) + pad, d), mk(n_pages, Hkv, page, d), mk(n_pages, Hkv, page, d)
    if outliers:
        Kp[..., 3] *= 20
        Q[..., 3] *= 4
        Vp[..., 5] *= 20
    q_start = np.concatenate([[0], np.cumsum(q)])
    return Q.to(DT[dt]), Kp.to(DT[dt]), Vp.to(DT[dt]), table, q_start, np.array(kv)


def _attn(case, causal, max_q=None, scale=None, Qd=None, Kd=None, Vd=None):
    Q, Kp, Vp, table, q_start, kv = case
    Hq, T, d = Q.shape
    O = torch.full((1, Hq, T, d), FILL, dtype=torch.float32, device=DEV)
    lse = torch.full((1, Hq, T), FILL, dtype=torch.float32, device=DEV)
    if max_q is None:
        max_q = max(int(q_start[-1]) and int(np.diff(q_start).max()), 0)
    fb.fedrag_paged_attn(Q.to(DEV) if Qd is None else Qd, Kp.to(DEV) if Kd is None else Kd, Vp.to(DEV) if Vd is None else Vd, i32(table),
                         i32(q_start), i32(kv), max_q, causal=causal, softmax_scale=scale, O_part=O, lse=lse)
    return O, lse


def _check(case, causal, what, max_q=None, scale=None, **kw):
    Q, Kp, Vp, table, q_start, kv = case
    O, lse = _attn(case, causal, max_q, scale, **kw)
    R.check_attn(O, lse, R.attn_ref(Q, Kp, Vp, table, q_start, kv, causal, Q.shape[2] ** -0.5 if scale is None else scale), FILL, what)


SETS = {
    # new rows and keys of each request
    "token": ([1], [1]),
    "token_page_edges": ([1] * 6, [15, 16, 17, 31, 32, 33]),
    "token_steps": ([1] * 8, [63, 64, 65, 127, 128, 129, 255, 257]),
    "token_none": ([1, 0, 1, 1, 0], [40, 55, 0, 3, 0]),
    "token_long": ([1, 1], [2500, 611]),
    "few": ([2, 3, 4, 1], [2, 40, 700, 9]),
    "chunk_edges": ([31, 32, 33, 17], [31, 64, 100, 17]),
    "chunk_64": ([63, 65], [200, 65]),
    "chunk_128": ([127, 129], [300, 129]),
    "chunk_long": ([40], [2100]),
    "more_rows_than_keys": ([20, 3, 70], [7, 0, 65]),
    "rows_that_see_nothing_of_runs": ([500, 2], [300, 700]),
    "mixed": ([1, 50, 0, 1, 5], [300, 50, 12, 17, 400]),
}


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("dt,d,page,Hq,Hkv", [("bf16", 128, 16, 8, 2), ("f16", 64, 32, 4, 4), ("f32", 64, 16, 4, 2), ("f32", 128, 64, 3, 1),
                                              ("bf16", 64, 128, 10, 2), ("f16", 128, 256, 7, 1)])
@pytest.mark.parametrize("name", list(SETS))
def test_attn(name, dt, d, page, Hq, Hkv, causal):
    q, kv = SETS[name]
    _check(_attn_case(q, kv, Hq, Hkv, d, page, dt, pad=3), causal, f"{name}/{dt}/{d}")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(16, 1), (17, 1), (33, 1), (40, 2), (3, 3), (71, 1)])
@pytest.mark.parametrize("q,kv", [([1, 1], [70, 333]), ([5, 30], [260, 30])], ids=["token", "chunk"])
def test_attn_head_layouts(dt, Hq, Hkv, q, kv):
    _check(_attn_case(q, kv, Hq, Hkv, 64, 16, dt), True, "heads")


@pytest.mark.parametrize("max_q", [0, 1, 4, 64, 10 ** 9])
def test_attn_any_expectation_of_the_longest(max_q):
    """max_q_len decides the kernels, not what they compute."""
    for dt in ("bf16", "f32"):
        _check(_attn_case([1, 70, 0, 3, 20], [100, 150, 7, 40, 900], 8, 2, 128, 32, dt), True, "max_q", max_q=max_q)


@pytest.mark.parametrize("B", [255, 256, 257, 600])
def test_attn_many_requests(B):
    rng = np.random.default_rng(B)
    kv = rng.integers(0, 40, B)
    q = np.minimum(rng.integers(0, 3, B), 2)
    q[B // 2], kv[B // 2] = 40, 45
    for dt in ("bf16", "f32"):
        _check(_attn_case(list(q), list(kv), 2, 1, 64, 16, dt), True, "many")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("q,kv,H", [([1100], [1100], 32), ([300], [300], 32), ([700, 500], [700, 900], 24), ([130], [140], 257), ([65], [65], 100)])
def test_attn_as_many_pieces_as_workgroups_fit(dt, q, kv, H):
    _check(_attn_case(q, kv, H, H, 64, 64, dt), True, dt)


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_attn_whole_tiles_beside_cut_ones(causal):
    """Tiles that fit a compute unit's part of the work stay whole; those of a long request are cut, and folded by the same launch."""
    _check(_attn_case([1000, 40, 3], [1500, 5000, 700], 24, 24, 64, 64, "bf16"), causal, "whole and cut")


@pytest.mark.parametrize("form", ["tokens", "fused", "broadcast"])
def test_attn_strided_queries(form):
    for dt in ("bf16", "f16", "f32"):
        case = list(_attn_case([1, 40, 3], [90, 60, 3], 8, 2, 128, 16, dt, pad=2))
        Q = case[0]
        if form == "tokens":
            Qd = Q.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
        elif form == "fused":
            x = torch.full((Q.shape[1], 12, 128), float("nan"), dtype=Q.dtype)
            x[:, 2:10] = Q.transpose(0, 1)
            Qd = x.to(DEV)[:, 2:10].transpose(0, 1)
        else:
            case[0] = Q[:1].expand(Q.shape).contiguous()
            Qd = Q[:1].to(DEV).expand(Q.shape)
        assert not Qd.is_contiguous()
        _check(case, True, form, Qd=Qd)


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f16", 64), ("f32", 64)])
def test_attn_interleaved_pages(dt, d):
    case = _attn_case([1, 33, 2], [90, 60, 700], 4, 2, d, 32, dt)
    both = torch.stack([case[1], case[2]], 1).to(DEV)
    _check(case, True, "interleaved", Kd=both[:, 0], Vd=both[:, 1])


@pytest.mark.parametrize("poison", ["nan", "inf", "lowest"])
@pytest.mark.parametrize("dt,d", [("bf16", 128), ("bf16", 64), ("f16", 128), ("f32", 128), ("f32", 64)])
def test_attn_hidden_tokens_do_not_matter(dt, d, poison):
    """Pages of nobody, the rest of a last page, and - causal - a chunk's later tokens hold anything."""
    bad = {"nan": float("nan"), "inf": float("inf"), "lowest": torch.finfo(DT[dt]).min}[poison]
    q, kv, page = [1, 40, 3, 150], [37, 80, 201, 150], 16
    Q, Kp, Vp, table, q_start, lens = _attn_case(q, kv, 4, 2, d, page, dt)
    clean = (Q, Kp.clone(), Vp.clone(), table, q_start, lens)
    used = np.zeros((Kp.shape[0], page), bool)
    for b, n in enumerate(kv):
        for t in range(n):
            used[table[b, t // page], t % page] = True
    hide = torch.from_numpy(~used)
    for x in (Kp, Vp):
        x.transpose(1, 2)[hide] = bad
    _check((Q, Kp, Vp, table, q_start, lens), True, f"behind/{poison}")
    _check((Q, Kp, Vp, table, q_start, lens), False, f"behind, no mask/{poison}")
    # the last five tokens of the second chunk, the second token of the third, some of the fourth: rows before them do not see them
    Kp, Vp = clean[1], clean[2]
    for b, ts in ((1, range(75, 80)), (2, (199,)), (3, (20, 64, 130))):
        for t in ts:
            Vp[table[b, t // page], :, t % page, ::3] = bad
            Kp[table[b, t // page], :, t % page, 5] = bad if poison != "lowest" else 0.0
    case = (Q, Kp, Vp, table, q_start, lens)
    O, lse = _attn(case, True)
    ref = R.attn_ref(*case, True, d ** -0.5)
    touched = np.zeros(sum(q), bool)
    for b, first in ((1, 75), (2, 199), (3, 20)):
        i = first - (kv[b] - q[b])
        touched[q_start[b] + i:q_start[b + 1]] = True
    hidden = tuple(x[:, ~touched] for x in ref[:4]) + (ref[4][~touched],)
    R.check_attn(O[:, :, torch.from_numpy(~touched).to(DEV)], lse[:, :, torch.from_numpy(~touched).to(DEV)], hidden, FILL, f"later/{poison}")
    if poison == "nan":  # and those that see it have it
        seen = O[0][:, torch.from_numpy(touched).to(DEV)][..., ::3]
        assert bool(torch.isnan(seen).all())


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f16", 64), ("f32", 128)])
def test_attn_pages_that_are_not_there(dt, d):
    """Table entries that name no page hold no tokens; neither do columns that the table does not have."""
    for q, kv in (([1, 1, 2, 1], [100, 300, 90, 40]), ([40, 20, 100, 17], [100, 300, 190, 40])):
        Q, Kp, Vp, table, q_start, lens = _attn_case(q, kv, 4, 2, d, 16, dt, more_columns=0)
        n = Kp.shape[0]
        table[0, 1], table[0, 6] = -1, n
        table[1, 3:9], table[1, 17] = 2 ** 31 - 1, -2 ** 31
        table[3, :] = n + 1
        for causal in (True, False):
            _check((Q, Kp, Vp, table, q_start, lens), causal, "holes")
            _check((Q, Kp, Vp, np.ascontiguousarray(table[:, :4]), q_start, lens), causal, "columns")
        _check((Q, Kp, Vp, table[:, :0], q_start, lens), True, "no columns")


def test_attn_lengths_beyond_the_tensors():
    """q_start above the rows there are and negative lengths are taken as the nearest that is possible."""
    for dt in ("bf16", "f32"):
        Q, Kp, Vp, table, q_start, lens = _attn_case([3, 40, 2], [30, 60, 9], 4, 2, 64, 16, dt)
        O, lse = _attn((Q, Kp, Vp, table, [-4, 3, 43, 2 ** 31 - 1], [30, 60, -8]), True, max_q=40)
        ref = R.attn_ref(Q, Kp, Vp, table, [0, 3, 43, 45], [30, 60, 0], True, 64 ** -0.5)
        R.check_attn(O, lse, ref, FILL, "beyond")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("columns,n_pages", [(0, 3), (4, 0), (0, 0)])
def test_attn_without_columns_or_pages(dt, columns, n_pages):
    """Lengths, but no table to say where, or no pool to point into: rows that see nothing."""
    for q, max_q in (([1, 1], 1), ([40, 0, 1], 0), ([200], 200)):
        T, B = sum(q), len(q)
        Q = torch.ones((8, T, 64), dtype=dt, device=DEV)
        pool = torch.empty((n_pages, 2, 16, 64), dtype=dt, device=DEV).fill_(float("nan"))
        O, lse = fb.fedrag_paged_attn(Q, pool, pool.clone(), i32(np.zeros((B, columns))), i32(np.concatenate([[0], np.cumsum(q)])),
                                      i32([500] * B), max_q, causal=max_q != 200, O_part=torch.full((1, 8, T, 64), 7.0, device=DEV),
                                      lse=torch.full((1, 8, T), 7.0, device=DEV))
        assert torch.all(O == 0) and torch.all(lse == -float("inf"))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attn_far_pages(dt):
    """Pages more than 2^32 bytes into a pool, K's and V's taking turns in it."""
    q, kv, page, d = [1, 50, 300], [700, 400, 300], 256, 64
    Q, Kp, Vp, table, q_start, lens = _attn_case(q, kv, 2, 1, d, page, dt)
    n = 2 ** 32 // (2 * page * d * Kp.element_size()) + 100
    pool = torch.empty((n, 2, 1, page, d), dtype=DT[dt], device=DEV)
    far = n - 1 - np.arange(Kp.shape[0])
    pool[far, 0], pool[far, 1] = Kp.to(DEV), Vp.to(DEV)
    ref = R.attn_ref(Q, Kp, Vp, table, q_start, lens, True, d ** -0.5)
    there = np.where(table >= 0, far[np.clip(table, 0, len(far) - 1)], -1)
    O, lse = fb.fedrag_paged_attn(Q.to(DEV), pool[:, 0], pool[:, 1], i32(there), i32(q_start), i32(lens), 300)
    R.check_attn(O[:, :, :sum(q)], lse[:, :, :sum(q)], tuple(x[:, :sum(q)] for x in ref[:4]) + (ref[4][:sum(q)],), FILL, "far")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_attn_outputs_beyond_four_gib(dt):
    """As many rows as make O pass 2^32 bytes, all with the same query: all of a head's rows are the first one's."""
    Hq, T, d = 64, 2 ** 32 // (64 * 64 * 4) + 7, 64
    g = torch.Generator().manual_seed(0)
    Q = torch.randn((Hq, 1, d), generator=g).to(dt).to(DEV).expand(Hq, T, d)
    pool = torch.randn((2, 3, 1, 16, d), generator=g).to(dt).to(DEV)
    O, lse = fb.fedrag_paged_attn(Q, pool[0], pool[1], i32([[2, 0]]), i32([0, T]), i32([21]), T, causal=False)
    first = slice(0, 1)
    ref = R.attn_ref(Q[:, first].cpu(), pool[0].cpu(), pool[1].cpu(), np.array([[2, 0]]), [0, 1], [21], False, d ** -0.5)
    R.check_attn(O[:, :, first], lse[:, :, first], ref, FILL, "first row")
    assert torch.equal(O, O[:, :, :1].expand_as(O)) and torch.equal(lse, lse[:, :, :1].expand_as(lse))


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f16", 128), ("bf16", 64), ("f32", 64)])
def test_attn_outliers(dt, d):
    """Logits of some hundreds and channels of 20 times the others."""
    _check(_attn_case([1, 60, 2], [1500, 200, 333], 8, 2, d, 16, dt, outliers=True), True, "outliers")
    _check(_attn_case([1, 60, 2], [1500, 200, 333], 8, 2, d, 16, dt), False, "scale", scale=1.0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attn_alone_and_in_a_batch(dt):
    """Twice the same call gives the same bits."""
    case = _attn_case([1, 50, 1], [3000, 600, 20], 8, 2, 128, 16, dt)
    a, b = _attn(case, True), _attn(case, True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
