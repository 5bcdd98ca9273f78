"""What the calls of a drafted step refuse, on the host, before anything is launched (made-up addresses are safe: every call fails)."""
import ctypes

import pytest
import torch

from paper_2605_25716_amd import binding as fb
from paper_2605_25716_amd import build as fbuild

A = 1 << 32  # far apart, so that only what a test moves together overlaps


@pytest.fixture(scope="module")
def lib():
    fbuild.build_library(force=False)
    return fb.load()


def P(x):
    return None if x is None else ctypes.c_void_p(x)


def shape(B=2, Hq=8, Hkv=2, d=128, dt=fb.BF16):
    return ctypes.byref(fb.Shape(B, Hq, Hkv, d, dt))


MAP = dict(batch=2, n_rows=40, words=1, q_start=A, kv=2 * A, parents=3 * A, mask=4 * A, positions=5 * A, flags=6 * A)


def map_call(lib, **kw):
    a = {**MAP, **kw}
    return lib.fedrag_tree_map(a["batch"], a["n_rows"], a["words"], P(a["q_start"]), P(a["kv"]), P(a["parents"]), P(a["mask"]),
                               P(a["positions"]), P(a["flags"]), None)


def test_map_refusals(lib):
    for k in ("q_start", "kv", "parents", "mask", "flags"):
        assert map_call(lib, **{k: None}) == fb.ERR_NULL, k
    for k in ("q_start", "kv", "parents", "positions", "flags"):
        assert map_call(lib, **{k: MAP[k] + 2}) == fb.ERR_ALIAS, k
    assert map_call(lib, mask=MAP["mask"] + 4) == fb.ERR_ALIAS
    for k, v in (("batch", -1), ("batch", 2 ** 31 - 1), ("n_rows", -1), ("n_rows", 2 ** 31 - 1), ("words", 0), ("words", -1), ("words", 65)):
        assert map_call(lib, **{k: v}) == fb.ERR_SHAPE, (k, v)
    for o in ("mask", "positions", "flags"):
        for other in MAP:
            if other not in ("batch", "n_rows", "words", o):
                assert map_call(lib, **{o: MAP[other]}) == fb.ERR_ALIAS, (o, other)
    assert map_call(lib, batch=0, n_rows=0, q_start=None, kv=None, parents=None, mask=None, positions=None, flags=None) == fb.OK


ATTN = dict(shape=None, n_rows=40, Q=A, hs=128, ts=1024, K=2 * A, V=3 * A, n_pages=10, ps=0, page=16, table=4 * A, columns=4, q_start=5 * A,
            kv=6 * A, mask=7 * A, words=1, max_q=8, scale=0.1, O=8 * A, lse=9 * A, ws=10 * A, ws_bytes=1 << 31)


def attn_call(lib, **kw):
    a = {**ATTN, **kw}
    rows = fb.Rows(a["Q"], a["hs"], a["ts"])
    cache = fb.PagedCache(a["K"], a["V"], a["n_pages"], a["ps"], a["page"])
    return lib.fedrag_paged_tree_attn(a["shape"] or shape(), a["n_rows"], ctypes.byref(rows), ctypes.byref(cache), P(a["table"]), a["columns"],
                                      P(a["q_start"]), P(a["kv"]), P(a["mask"]), a["words"], a["max_q"], a["scale"], P(a["O"]), P(a["lse"]),
                                      P(a["ws"]), a["ws_bytes"], None)


def test_attn_refusals(lib):
    for k in ("Q", "K", "V", "table", "q_start", "kv", "mask", "O", "lse"):
        assert attn_call(lib, **{k: None}) == fb.ERR_NULL, k
    assert lib.fedrag_paged_tree_attn(None, 4, None, None, None, 0, None, None, None, 1, 0, 0.1, None, None, None, 0, None) == fb.ERR_NULL
    for k, v in (("n_rows", -1), ("n_rows", 2 ** 31 - 1), ("columns", -1), ("columns", 1 << 27), ("max_q", -1), ("n_pages", -1), ("ps", -8),
                 ("hs", -8), ("ts", 1 << 62), ("scale", 0.0), ("scale", float("nan")), ("words", 0), ("words", 65), ("words", -3)):
        assert attn_call(lib, **{k: v}) == fb.ERR_SHAPE, (k, v)
    assert attn_call(lib, page=24) == fb.ERR_UNSUPPORTED
    assert attn_call(lib, shape=shape(d=96)) == fb.ERR_UNSUPPORTED
    assert attn_call(lib, shape=shape(dt=5)) == fb.ERR_UNSUPPORTED
    assert attn_call(lib, shape=shape(Hq=7)) == fb.ERR_SHAPE
    for k in ("Q", "K", "V", "O", "ws"):
        assert attn_call(lib, **{k: ATTN[k] + 8}) == fb.ERR_ALIAS, k
    for k in ("table", "q_start", "kv", "lse"):
        assert attn_call(lib, **{k: ATTN[k] + 2}) == fb.ERR_ALIAS, k
    assert attn_call(lib, mask=ATTN["mask"] + 4) == fb.ERR_ALIAS
    for k in ("Q", "K", "V", "table", "q_start", "kv", "mask", "lse"):
        assert attn_call(lib, O=ATTN[k]) == fb.ERR_ALIAS, k
        if k != "lse":
            assert attn_call(lib, lse=ATTN[k]) == fb.ERR_ALIAS, k
    assert attn_call(lib, n_rows=0, Q=None, O=None, lse=None, q_start=None, kv=None, mask=None) == fb.OK
    assert attn_call(lib, shape=shape(B=0), Q=None, O=None, lse=None, q_start=None, kv=None, mask=None) == fb.OK


def test_attn_workspace(lib):
    big = dict(shape=shape(B=2, Hq=32, Hkv=8), n_rows=12, columns=4096, hs=128, ts=4096, max_q=6)
    need = lib.fedrag_paged_tree_attn_workspace_bytes(big["shape"], 12, 4096, 16, 6)
    assert need > 0
    assert attn_call(lib, **big, ws=None) == fb.ERR_WORKSPACE
    assert attn_call(lib, **big, ws_bytes=need - 1) == fb.ERR_WORKSPACE
    for k in ("Q", "K", "V", "table", "q_start", "kv", "mask", "O", "lse"):
        assert attn_call(lib, **big, ws=ATTN[k]) == fb.ERR_ALIAS, k
    for bad in ((shape(d=96), 2, 4, 16, 1), (shape(), -1, 4, 16, 1), (shape(), 2, -4, 16, 1), (shape(), 2, 4, 24, 1), (shape(), 2, 4, 16, -1),
                (None, 2, 4, 16, 1), (shape(), 2 ** 31 - 1, 4, 16, 1)):
        assert lib.fedrag_paged_tree_attn_workspace_bytes(*bad) == 0


VERIFY = dict(batch=2, n_rows=10, vocab=70000, dtype=fb.F32, q_start=A, parents=2 * A, tokens=3 * A, target=4 * A, ts=70000, draft=5 * A, ds=70000, u=6 * A,
              u_next=7 * A, most=4, kept=8 * A, n_kept=9 * A, next=10 * A, ws=11 * A, ws_bytes=1 << 20)


def verify_call(lib, **kw):
    a = {**VERIFY, **kw}
    return lib.fedrag_tree_verify(a["batch"], a["n_rows"], a["vocab"], a["dtype"], P(a["q_start"]), P(a["parents"]), P(a["tokens"]), P(a["target"]),
                                  a["ts"], P(a["draft"]), a["ds"], P(a["u"]), P(a["u_next"]), a["most"], P(a["kept"]), P(a["n_kept"]), P(a["next"]),
                                  P(a["ws"]), a["ws_bytes"], None)


def test_verify_refusals(lib):
    for k in ("q_start", "parents", "tokens", "target", "u", "u_next", "kept", "n_kept", "next"):
        assert verify_call(lib, **{k: None}) == fb.ERR_NULL, k
    for k, v in (("batch", -1), ("batch", 65536), ("n_rows", -1), ("n_rows", 2 ** 31 - 1), ("vocab", 0), ("vocab", (1 << 20) + 1), ("ts", 69999),
                 ("ds", 69999), ("most", 0), ("most", 1 << 31), ("ts", 1 << 61), ("ds", 1 << 61)):
        assert verify_call(lib, **{k: v}) == fb.ERR_SHAPE, (k, v)
    assert verify_call(lib, dtype=3) == fb.ERR_UNSUPPORTED
    need = lib.fedrag_tree_verify_workspace_bytes(2, 70000, fb.F32)
    assert need > 0 and verify_call(lib, ws=None) == fb.ERR_WORKSPACE and verify_call(lib, ws_bytes=need - 1) == fb.ERR_WORKSPACE
    for k in ("q_start", "parents", "tokens", "target", "draft", "kept", "n_kept", "next"):
        assert verify_call(lib, **{k: VERIFY[k] + 2}) == fb.ERR_ALIAS, k
    for k in ("u", "u_next", "ws"):
        assert verify_call(lib, **{k: VERIFY[k] + 4}) == fb.ERR_ALIAS, k
    assert verify_call(lib, dtype=fb.BF16, target=VERIFY["target"] + 1) == fb.ERR_ALIAS
    for o in ("kept", "n_kept", "next", "ws"):
        for other in ("q_start", "parents", "tokens", "target", "draft", "u", "u_next", "kept", "n_kept", "next", "ws"):
            if o != other:
                assert verify_call(lib, **{o: VERIFY[other]}) == fb.ERR_ALIAS, (o, other)
    assert verify_call(lib, batch=0, q_start=None, u_next=None, kept=None, n_kept=None, next=None) == fb.OK
    for dtype, most in ((fb.F32, 32768), (fb.BF16, 65536), (fb.F16, 65536)):  # what one workgroup has in its registers
        for vocab, some in ((1, True), (3 if dtype == fb.F32 else 7, True), (8, False), (500, False), (most, False), (most + 1, True)):
            assert (lib.fedrag_tree_verify_workspace_bytes(2, vocab, dtype) > 0) == some, (dtype, vocab)
    for bad in ((-1, 70000, fb.F32), (2, 0, fb.F32), (65536, 70000, fb.F32), (2, (1 << 20) + 1, fb.F32), (2, 70000, 3)):
        assert lib.fedrag_tree_verify_workspace_bytes(*bad) == 0


KEEP = dict(shape=None, n_caches=2, K=(A, 2 * A), V=(3 * A, 4 * A), n_pages=(10, 12), ps=(0, 0), page=(16, 16), table=5 * A, columns=4, q_start=6 * A,
            kv=7 * A, kept=8 * A, most=4, n_kept=9 * A)


def keep_call(lib, **kw):
    a = {**KEEP, **kw}
    caches = (fb.PagedCache * len(a["K"]))(*[fb.PagedCache(*x) for x in zip(a["K"], a["V"], a["n_pages"], a["ps"], a["page"])])
    return lib.fedrag_paged_keep(a["shape"] or shape(), a["n_caches"], None if a.get("none") else caches, P(a["table"]), a["columns"], P(a["q_start"]),
                                 P(a["kv"]), P(a["kept"]), a["most"], P(a["n_kept"]), None)


def test_keep_refusals(lib):
    for k in ("table", "q_start", "kv", "kept", "n_kept"):
        assert keep_call(lib, **{k: None}) == fb.ERR_NULL, k
        assert keep_call(lib, **{k: KEEP[k] + 2}) == fb.ERR_ALIAS, k
        assert keep_call(lib, **{k: KEEP["V"][1] + 64}) == fb.ERR_ALIAS, k
    assert keep_call(lib, none=True) == fb.ERR_NULL
    assert keep_call(lib, K=(A, None)) == fb.ERR_NULL
    for k, v in (("n_caches", 0), ("n_caches", -1), ("n_caches", 65), ("most", -1), ("most", 1 << 31), ("columns", -1), ("columns", 1 << 27),
                 ("n_pages", (10, -1)), ("ps", (0, 8)), ("page", (16, 32)), ("shape", shape(B=-1)), ("shape", shape(B=1 << 19)), ("shape", shape(Hq=7))):
        assert keep_call(lib, **{k: v}) == fb.ERR_SHAPE, (k, v)
    assert keep_call(lib, page=(16, 24)) == fb.ERR_UNSUPPORTED and keep_call(lib, shape=shape(d=32)) == fb.ERR_UNSUPPORTED
    assert keep_call(lib, V=(3 * A, 4 * A + 8)) == fb.ERR_ALIAS
    page = 2 * 16 * 128 * 2  # bytes of a page
    for K, V in (((A, A), (3 * A, 4 * A)), ((A, 2 * A), (3 * A, A)), ((A, 2 * A), (2 * A + 16, 4 * A)), ((A, A + 9 * page), (3 * A, 4 * A))):
        assert keep_call(lib, K=K, V=V) == fb.ERR_ALIAS, (K, V)
    assert keep_call(lib, most=0, kept=None) == fb.OK and keep_call(lib, shape=shape(B=0)) == fb.OK


def test_caches_that_take_turns_in_one_tensor(lib):
    """Layers' K and V pages interleaved: apart, though their extents overlap.  (Everything is in order, so the call gets as far as an
    argument that is refused later than the pages.)"""
    page = 2 * 16 * 128 * 2
    turns = dict(K=(A, A + 2 * page), V=(A + page, A + 3 * page), ps=(4 * page // 2, 4 * page // 2), n_pages=(10, 10))
    assert keep_call(lib, **turns, shape=shape(B=0)) == fb.OK
    assert keep_call(lib, **{**turns, "V": (A + page, A + 3 * page + 16)}) == fb.ERR_ALIAS


TRIM = dict(batch=2, page=16, columns=4, kv=A, q_start=2 * A, n_kept=3 * A, table=4 * A, free=5 * A, n_free=9, count=6 * A, lens=7 * A, left=8 * A,
            flags=9 * A)


def trim_call(lib, **kw):
    a = {**TRIM, **kw}
    return lib.fedrag_paged_trim(a["batch"], a["page"], a["columns"], P(a["kv"]), P(a["q_start"]), P(a["n_kept"]), P(a["table"]), P(a["free"]),
                                 a["n_free"], P(a["count"]), P(a["lens"]), P(a["left"]), P(a["flags"]), None)


def test_trim_refusals(lib):
    for k in ("kv", "n_kept", "table", "free", "count", "lens", "left", "flags"):
        assert trim_call(lib, **{k: None}) == fb.ERR_NULL, k
    for k in ("kv", "q_start", "n_kept", "table", "free", "count", "lens", "left", "flags"):
        assert trim_call(lib, **{k: TRIM[k] + 2}) == fb.ERR_ALIAS, k
    for k, v in (("batch", -1), ("batch", 2 ** 31 - 1), ("columns", -1), ("columns", 1 << 31), ("n_free", -1), ("n_free", 1 << 31)):
        assert trim_call(lib, **{k: v}) == fb.ERR_SHAPE, (k, v)
    assert trim_call(lib, page=48) == fb.ERR_UNSUPPORTED
    for o in ("free", "lens", "left", "flags"):
        for other in ("kv", "q_start", "n_kept", "table", "free", "count", "lens", "left", "flags"):
            if o != other and (o, other) not in (("lens", "kv"), ("left", "count")):
                assert trim_call(lib, **{o: TRIM[other]}) == fb.ERR_ALIAS, (o, other)
    assert trim_call(lib, lens=TRIM["kv"] + 4) == fb.ERR_ALIAS  # in place, but shifted


def test_binding_refuses_host_tensors():
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.float64)
    pages, p = torch.zeros((2, 1, 16, 64)), torch.zeros((4, 10))
    for call in (lambda: fb.fedrag_tree_map(i, i, i, 1), lambda: fb.fedrag_tree_verify(p, i, i, i, f, f),
                 lambda: fb.fedrag_paged_tree_attn(pages[0], pages, pages, i.view(2, 2), i, i, i.view(2, 2)),
                 lambda: fb.fedrag_paged_keep([(pages, pages)], i.view(2, 2), i, i, i.view(2, 2), i),
                 lambda: fb.fedrag_paged_trim(i, i, i.view(2, 2), i, i, 16), lambda: fb.fedrag_paged_keep([], i, i, i, i, i)):
        with pytest.raises(ValueError):
            call()


def test_attn_workspace_has_a_bound(lib):
    """What a caller may set aside once for all its calls: 1024 partials of 128 rows of d + 1 numbers, and 512 of 32 rows."""
    assert (1024 * 128 + 512 * 32) * 129 * 4 <= 73 * 2 ** 20
    for B, T in [(B, T) for B in (1, 7, 64, 1000) for T in (1, 3, 17, 64, 300, 1000, 5000, 70000)]:
        for Hkv, G in ((1, 1), (1, 16), (8, 4), (33, 2)):
            for d, dtype in ((64, fb.F32), (128, fb.F32), (128, fb.BF16)):
                for columns in (1, 9, 100, 3000, 40000):
                    for max_q in (0, 1, 5, 12, T):
                        need = lib.fedrag_paged_tree_attn_workspace_bytes(shape(B=B, Hq=G * Hkv, Hkv=Hkv, d=d, dt=dtype), T, columns, 16, max_q)
                        assert need <= 73 * 2 ** 20, (B, T, Hkv, G, d, dtype, columns, max_q)
