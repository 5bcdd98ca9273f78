"""What the paged calls refuse, on the host, before anything is launched (made-up addresses are safe: every call fails)."""
import ctypes
import os
import subprocess

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


MAP = dict(batch=2, n_rows=40, page=16, columns=4, cached=A, new=2 * A, free=3 * A, n_free=9, count=4 * A, table=5 * A, q_start=6 * A,
           kv=7 * A, slots=8 * A, positions=9 * A, left=10 * A, flags=11 * A)


def map_call(lib, **kw):
    a = {**MAP, **kw}
    return lib.fedrag_paged_map(a["batch"], a["n_rows"], a["page"], a["columns"], P(a["cached"]), P(a["new"]), P(a["free"]), a["n_free"],
                                P(a["count"]), P(a["table"]), P(a["q_start"]), P(a["kv"]), P(a["slots"]), P(a["positions"]), P(a["left"]),
                                P(a["flags"]), None)


def test_map_refusals(lib):
    for k in ("cached", "new", "free", "count", "table", "q_start", "kv", "slots", "left", "flags"):
        assert map_call(lib, **{k: None}) == fb.ERR_NULL, k
    for k in ("cached", "new", "free", "count", "table", "q_start", "kv", "positions", "left", "flags"):
        assert map_call(lib, **{k: MAP[k] + 2}) == fb.ERR_ALIAS, k
    assert map_call(lib, slots=MAP["slots"] + 4) == fb.ERR_ALIAS
    for k, v in (("batch", -1), ("n_rows", -1), ("n_rows", 1 << 31), ("columns", -1), ("columns", 1 << 31), ("n_free", -1), ("n_free", 1 << 31)):
        assert map_call(lib, **{k: v}) == fb.ERR_SHAPE, (k, v)
    for page in (0, 8, 24, 48, 512, -16):
        assert map_call(lib, page=page) == fb.ERR_UNSUPPORTED
    # what is written overlaps nothing but what it may be
    outs = ("table", "q_start", "kv", "slots", "positions", "left", "flags")
    for o in outs:
        for other in ("cached", "new", "free", "count") + outs:
            if o != other and (o, other) not in (("kv", "cached"), ("left", "count")):
                assert map_call(lib, **{o: MAP[other]}) == fb.ERR_ALIAS, (o, other)
    assert map_call(lib, kv=MAP["cached"] + 4) == fb.ERR_ALIAS  # in place, but shifted
    assert map_call(lib, batch=3, cached=A, new=A + 4, kv=A + 8) == fb.ERR_ALIAS


ATTN = dict(shape=None, n_rows=40, Q=A, hs=128, ts=1024, K=2 * A, V=3 * A, n_pages=10, ps=0, page=16, table=4 * A, columns=4, q_start=5 * A,
            kv=6 * A, max_q=8, causal=1, scale=0.1, O=7 * A, lse=8 * A, ws=9 * A, ws_bytes=1 << 31)


def attn_call(lib, **kw):
    a = {**ATTN, **kw}
    rows = fb.Rows(a["Q"], a["hs"], a["ts"])
    cache = fb.PagedCache(a["K"], a["V"], a["n_pages"], a["ps"], a["page"])
    return lib.fedrag_paged_attn(a["shape"] or shape(), a["n_rows"], None if a["Q"] == "none" else ctypes.byref(rows),
                                 None if a["K"] == "none" else ctypes.byref(cache), P(a["table"]), a["columns"], P(a["q_start"]), P(a["kv"]),
                                 a["max_q"], a["causal"], a["scale"], P(a["O"]), P(a["lse"]), P(a["ws"]), a["ws_bytes"], None)


def test_attn_refusals(lib):
    for k in ("Q", "K", "V", "table", "q_start", "kv", "O", "lse"):
        assert attn_call(lib, **{k: None}) == fb.ERR_NULL, k
    assert lib.fedrag_paged_attn(shape(), 4, None, None, None, 0, None, None, 0, 0, 0.1, None, None, None, 0, None) == fb.ERR_NULL
    assert lib.fedrag_paged_attn(None, 4, None, None, None, 0, None, None, 0, 0, 0.1, None, None, None, 0, None) == fb.ERR_NULL
    for k, v in (("n_rows", -1), ("n_rows", 1 << 31), ("columns", -1), ("columns", 1 << 31), ("columns", 1 << 27), ("max_q", -1), ("n_pages", -1),
                 ("n_pages", 1 << 31), ("ps", -8), ("ps", 16 * 128 * 2 - 8), ("hs", -8), ("ts", -8), ("hs", 1 << 62), ("ts", 1 << 62),
                 ("scale", 0.0), ("scale", -1.0), ("scale", float("inf")), ("scale", float("nan"))):
        assert attn_call(lib, **{k: v}) == fb.ERR_SHAPE, (k, v)
    for page in (0, 8, 17, 48, 512):
        assert attn_call(lib, page=page) == fb.ERR_UNSUPPORTED
    assert attn_call(lib, shape=shape(d=96)) == fb.ERR_UNSUPPORTED
    assert attn_call(lib, shape=shape(dt=5)) == fb.ERR_UNSUPPORTED
    assert attn_call(lib, shape=shape(Hq=7)) == fb.ERR_SHAPE
    assert attn_call(lib, shape=shape(B=-1)) == fb.ERR_SHAPE
    for k in ("Q", "K", "V", "O", "ws"):
        assert attn_call(lib, **{k: ATTN[k] + 8}) == fb.ERR_ALIAS, k
    for k in ("table", "q_start", "kv", "lse"):
        assert attn_call(lib, **{k: ATTN[k] + 2}) == fb.ERR_ALIAS, k
    for k, v in (("hs", 4), ("ts", 1020), ("ps", 16 * 128 * 2 + 4)):
        assert attn_call(lib, **{k: v}) == fb.ERR_ALIAS, k
    for k in ("Q", "K", "V", "table", "q_start", "kv", "lse"):
        assert attn_call(lib, O=ATTN[k]) == fb.ERR_ALIAS, k
        if k != "lse":
            assert attn_call(lib, lse=ATTN[k]) == fb.ERR_ALIAS, k
    # nothing to do: no rows, or no requests
    assert attn_call(lib, n_rows=0, Q=None, O=None, lse=None, q_start=None, kv=None) == fb.OK
    assert attn_call(lib, shape=shape(B=0), Q=None, O=None, lse=None, q_start=None, kv=None) == fb.OK


def test_attn_workspace(lib):
    big = dict(shape=shape(B=2, Hq=32, Hkv=8), n_rows=2, columns=4096, hs=128, ts=4096, max_q=1)
    need = lib.fedrag_paged_attn_workspace_bytes(big["shape"], 2, 4096, 16, 1)
    if need:
        assert attn_call(lib, **big, ws=None) == fb.ERR_WORKSPACE
        assert attn_call(lib, **big, ws_bytes=need - 1) == fb.ERR_WORKSPACE
        for k in ("Q", "K", "V", "table", "q_start", "kv", "O", "lse"):
            assert attn_call(lib, **big, ws=ATTN[k]) == fb.ERR_ALIAS, k
    for bad in ((shape(d=96), 2, 4, 16, 1), (shape(), -1, 4, 16, 1), (shape(), 2, -4, 16, 1), (shape(), 2, 4, 24, 1), (shape(), 2, 4, 16, -1),
                (None, 2, 4, 16, 1)):
        assert lib.fedrag_paged_attn_workspace_bytes(*bad) == 0


def test_attn_workspace_has_a_bound(lib):
    """What a caller may set aside once for all its calls."""
    sizes = [(B, T) for B in (1, 7, 64, 1000) for T in (1, 3, 17, 64, 300, 1000, 5000, 70000)]
    for B, T in sizes:
        for Hkv, G in ((1, 1), (1, 16), (8, 4), (33, 2)):
            for d, dtype in ((64, fb.F32), (128, fb.F32), (128, fb.BF16)):
                for columns in (1, 9, 100, 3000, 40000):
                    for max_q in (0, 1, 5, T):
                        need = lib.fedrag_paged_attn_workspace_bytes(shape(B=B, Hq=G * Hkv, Hkv=Hkv, d=d, dt=dtype), T, columns, 16, max_q)
                        assert need <= 69 * 2 ** 20, (B, T, Hkv, G, d, dtype, columns, max_q)


WRITE = dict(shape=None, n_rows=40, K=A, V=2 * A, hs=128, ts=1024, slots=3 * A, Kp=4 * A, Vp=5 * A, n_pages=10, ps=0, page=16)


def write_call(lib, **kw):
    a = {**WRITE, **kw}
    k, v = fb.Rows(a["K"], a["hs"], a["ts"]), fb.Rows(a["V"], 128, 1024)
    cache = fb.PagedCache(a["Kp"], a["Vp"], a["n_pages"], a["ps"], a["page"])
    return lib.fedrag_paged_write(a["shape"] or shape(), a["n_rows"], ctypes.byref(k), ctypes.byref(v), P(a["slots"]), ctypes.byref(cache), None)


def test_write_refusals(lib):
    for k in ("K", "V", "slots", "Kp", "Vp"):
        assert write_call(lib, **{k: None}) == fb.ERR_NULL, k
    assert lib.fedrag_paged_write(shape(), 4, None, None, P(A), None, None) == fb.ERR_NULL
    for k, v in (("n_rows", -1), ("n_rows", 1 << 31), ("n_pages", -1), ("hs", -8), ("ts", -8), ("ps", 8), ("ts", 1 << 62)):
        assert write_call(lib, **{k: v}) == fb.ERR_SHAPE, (k, v)
    for k in ("K", "V", "Kp", "Vp"):
        assert write_call(lib, **{k: WRITE[k] + 8}) == fb.ERR_ALIAS, k
    assert write_call(lib, slots=WRITE["slots"] + 4) == fb.ERR_ALIAS
    assert write_call(lib, hs=132) == fb.ERR_ALIAS
    for k in ("K", "V", "slots"):
        assert write_call(lib, Kp=WRITE[k]) == fb.ERR_ALIAS
        assert write_call(lib, Vp=WRITE[k]) == fb.ERR_ALIAS
    assert write_call(lib, Vp=WRITE["Kp"]) == fb.ERR_ALIAS
    block = 2 * 16 * 128 * 2  # bytes
    assert write_call(lib, Vp=WRITE["Kp"] + block, ps=2 * block // 2 - 8) == fb.ERR_ALIAS  # a page of V begins where one of K ends, the next too early
    assert write_call(lib, Vp=WRITE["Kp"] + block, ps=0) == fb.ERR_ALIAS
    assert write_call(lib, n_rows=0, K=None, V=None, slots=None) == fb.OK
    assert write_call(lib, n_pages=0, Kp=None, Vp=None) == fb.OK


def test_binding_refuses_host_tensors():
    z = torch.zeros
    with pytest.raises(ValueError):
        fb.fedrag_paged_map(z(1, dtype=torch.int32), z(1, dtype=torch.int32), z((1, 2), dtype=torch.int32), z(4, dtype=torch.int32),
                            z(1, dtype=torch.int32), 16, 4)
    with pytest.raises(ValueError):
        fb.fedrag_paged_write(z(2, 3, 64), z(2, 3, 64), z(3, dtype=torch.int64), z(4, 2, 16, 64), z(4, 2, 16, 64))
    with pytest.raises(ValueError):
        fb.fedrag_paged_attn(z(2, 3, 64), z(4, 2, 16, 64), z(4, 2, 16, 64), z((1, 2), dtype=torch.int32), z(2, dtype=torch.int32),
                             z(1, dtype=torch.int32))


def test_pages_have_memory_of_their_own():
    """A stride of 0 between pages is the struct's word for pages side by side, which those of an expanded tensor are not."""
    for pool in (torch.zeros((1, 2, 16, 64)).expand(4, 2, 16, 64), torch.zeros((2, 16, 64), dtype=torch.bfloat16).expand(4, 2, 16, 64)):
        with pytest.raises(ValueError):
            fb._page_stride(pool.shape, pool.stride())
    both = torch.zeros((4, 2, 2, 16, 64))
    for pool, want in ((both[0, 0][None].expand(1, 2, 16, 64), 0), (both[:, 0], 4096), (both[:, 0].contiguous(), 2048), (both[:0, 0], 0)):
        assert fb._page_stride(pool.shape, pool.stride()) == want


def test_most_requests(lib):
    """What is reckoned with requests a lane, rounded up, stays in 32 bits."""
    most, far = 2 ** 31 - 1 - 255, 1 << 40  # (their arrays pass the distance of the others)
    addresses = {k: far * (i + 1) for i, k in enumerate(("cached", "new", "free", "count", "table", "q_start", "kv", "slots", "positions", "left", "flags"))}
    for batch in (most + 1, 2 ** 31 - 1):
        assert map_call(lib, **addresses, batch=batch) == fb.ERR_SHAPE
        assert attn_call(lib, shape=shape(B=batch), q_start=far, kv=2 * far, table=3 * far) == fb.ERR_SHAPE
        assert lib.fedrag_paged_attn_workspace_bytes(shape(B=batch), 40, 400, 16, 8) == 0
    # one less goes on to what comes behind: that the tables overlap, or the scratch is missing
    assert map_call(lib, **{**addresses, "new": addresses["kv"]}, batch=most) == fb.ERR_ALIAS
    assert attn_call(lib, shape=shape(B=most), q_start=far, kv=2 * far, table=3 * far, columns=400, ws=None) == fb.ERR_WORKSPACE


def test_what_a_launch_holds(lib):
    """Sizes that no launch holds are refused as sizes, and need no scratch."""
    far = 1 << 44
    at = dict(Q=far, O=2 * far, lse=3 * far, ws=4 * far, q_start=5 * far, kv=6 * far, table=7 * far)
    for sizes, n_rows, max_q in ((dict(B=2, Hq=64, Hkv=1, d=64), 1 << 26, 0), (dict(B=2, Hq=64, Hkv=1, d=64), 1 << 25, 7),
                                 (dict(B=1 << 21, Hq=8, Hkv=8, d=64, dt=fb.F32), 1 << 21, 1)):
        kw = dict(at, shape=shape(**sizes), n_rows=n_rows, max_q=max_q, hs=0, ts=64, columns=400)
        assert attn_call(lib, **kw) == fb.ERR_SHAPE, sizes
        assert lib.fedrag_paged_attn_workspace_bytes(shape(**sizes), n_rows, 400, 16, max_q) == 0
        fewer = n_rows // 4
        assert attn_call(lib, **dict(kw, n_rows=fewer, ws=None)) == fb.ERR_WORKSPACE, sizes
        assert lib.fedrag_paged_attn_workspace_bytes(shape(**sizes), fewer, 400, 16, max_q) > 0
    at = dict(K=far, V=2 * far, slots=3 * far, Kp=4 * far, Vp=5 * far)
    assert write_call(lib, **at, shape=shape(Hq=8, Hkv=8, d=128), n_rows=1 << 24) == fb.ERR_SHAPE
    assert write_call(lib, **at, shape=shape(Hq=65536, Hkv=65536, d=128), n_rows=1) == fb.ERR_SHAPE


def test_host_paths_under_sanitizers():
    """The host side of the paged calls with the library's host code under address and undefined-behaviour sanitizers, over 200000 random
    sizes and those at the ends; no call reaches a launch."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = fbuild.build_host_check(os.path.join(root, "tests", "c", "paged_host_paths.c"))
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, f"{res.stdout[-3000:]}\n{res.stderr[-3000:]}"
    assert "paged host paths ok" in res.stdout


def test_structs_match_the_header(tmp_path):
    """The binding's structs have the header's sizes and offsets."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "fedrag.h"\nint main(void) { printf("%zu %zu %zu %zu %zu\\n", sizeof(fedrag_paged_cache), '
                   'offsetof(fedrag_paged_cache, page_stride), offsetof(fedrag_paged_cache, page_tokens), sizeof(fedrag_rows), '
                   'offsetof(fedrag_rows, token_stride)); return 0; }\n')
    exe = str(tmp_path / "sizes")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(fb.PagedCache), fb.PagedCache.page_stride.offset, fb.PagedCache.page_tokens.offset, ctypes.sizeof(fb.Rows),
                   fb.Rows.token_stride.offset]
