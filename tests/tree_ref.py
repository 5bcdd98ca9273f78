"""Plain 64-bit statements of a drafted step's calls.

Attention: paged_ref's, with a row's own mask in place of the causal one, and its tolerances (the kernels' sums are of the same lengths
and in the same number of steps).  Everything else is whole numbers or copies, and has to be equal: the verification's weights are
counted in units of 2^-43, its products and differences are those of IEEE double precision, which numpy's are too.
"""
import numpy as np
import torch

import paged_ref as R

UNIT = 2.0 ** 43


def trees(rng, sizes, shape="tree"):
    """Parents within each request, node 0 without one."""
    out = []
    for n in sizes:
        for i in range(n):
            if i == 0:
                out.append(-1)
            elif shape == "chain":
                out.append(i - 1)
            elif shape == "star":
                out.append(0)
            elif shape == "forest":
                out.append(int(rng.integers(-1, i)))
            else:
                out.append(int(rng.integers(max(0, i - 4), i)))
    return np.array(out, dtype=np.int64)


def starts(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)


def map_ref(parents, q_start, kv, words, T):
    """(masks [T][words] of Python integers, positions, flags)"""
    masks, positions, flags = [[0] * words for _ in range(T)], [-1] * T, []
    for b in range(len(kv)):
        s, e = (min(max(int(x), 0), T) for x in q_start[b:b + 2])
        n = max(e - s, 0)
        flag = 2 if n > 64 * words else 0
        seen, depth = [], []
        for i in range(n):
            p = int(parents[s + i])
            if not -1 <= p < i:
                flag |= 1
                p = -1
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
            depth.append(depth[p] + 1 if p >= 0 else 0)
            masks[s + i] = [seen[i] >> 64 * w & (1 << 64) - 1 for w in range(words)]
            positions[s + i] = max(int(kv[b]), 0) - n + depth[i]
        flags.append(flag)
    return masks, positions, flags


def signed(masks):
    """Words as the int64 that hold their bits."""
    return np.array([[w - (1 << 64) if w >> 63 else w for w in row] for row in masks], dtype=np.int64).reshape(len(masks), -1)


def attn_ref(Q, Kp, Vp, table, q_start, kv_lens, mask, scale):
    """paged_ref.attn_ref's answer for rows with masks (int64 [T, words]); everything on the CPU"""
    Q64, K64, V64 = (x.double().numpy() for x in (Q, Kp, Vp))
    Hq, T, d = Q64.shape
    n_pages, Hkv, P, _ = K64.shape
    table, q_start, kv_lens = (np.asarray(x, dtype=np.int64) for x in (table, q_start, kv_lens))
    two_terms = 2.0 ** -16 if Q.dtype != torch.float32 else 0.0
    O, lse = np.zeros((Hq, T, d)), np.full((Hq, T), -np.inf)
    tol_o, tol_l = np.zeros((Hq, T, d)), np.zeros((Hq, T))
    written = np.zeros(T, bool)
    for b in range(table.shape[0]):
        s, e = (min(max(int(x), 0), T) for x in q_start[b:b + 2])
        n, kv = e - s, max(int(kv_lens[b]), 0)
        if n <= 0:
            continue
        written[s:e] = True
        key = np.arange(min(kv, table.shape[1] * P))
        ids = table[b][key // P]
        there = (ids >= 0) & (ids < n_pages)
        key, ids = key[there], ids[there]
        node = key - (kv - n)
        for i in range(n):
            word = np.clip(node // 64, 0, mask.shape[1] - 1)
            bit = mask[s + i][word] >> (node % 64) & 1
            sees = (node < 0) | ((node < 64 * mask.shape[1]) & (bit == 1))
            if not sees.any():
                continue
            for h in range(Hq):
                k, v = K64[ids[sees], h // (Hq // Hkv), key[sees] % P], V64[ids[sees], h // (Hq // Hkv), key[sees] % P]
                q = Q64[h, s + i]
                with np.errstate(invalid="ignore"):
                    x = (k @ q) * scale
                    m = x.max()
                    p = np.exp(x - m)
                    total = p.sum()
                    O[h, s + i] = p @ v / total
                    lse[h, s + i] = m + np.log(total)
                    off = 16 * R.U * scale * (np.abs(k) @ np.abs(q)).max() + 8 * R.U * np.sqrt(len(k))
                    tol_o[h, s + i] = (2 * off + 2.0 ** -21 + two_terms) * (p @ np.abs(v) / total)
                    tol_l[h, s + i] = off + 4 * R.U * abs(lse[h, s + i]) + 2.0 ** -20
    return O, lse, tol_o, tol_l, written


def _values(x):
    return np.clip(np.nan_to_num(x.double().numpy(), nan=0.0, posinf=1.0, neginf=0.0), 0.0, 1.0)


def _units(r):
    return np.rint(np.maximum(r, 0.0) * UNIT).astype(np.int64)


def verify_ref(target, draft, tokens, parents, q_start, u, u_next, max_kept):
    """(kept, n_kept, next_token) by the header's rules, one child at a time; tensors on the CPU"""
    T, V = target.shape
    B = len(q_start) - 1
    p_all = _values(target)
    q_all = None if draft is None else _values(draft)
    kept, n_kept, after = np.zeros((B, max_kept), np.int64), np.zeros(B, np.int64), np.full(B, -1, np.int64)
    below_one = np.nextafter(1.0, 0.0)
    rand = lambda x: min(max(float(x), 0.0), below_one) if x == x else 0.0  # noqa: E731
    for b in range(B):
        s, e = (min(max(int(x), 0), T) for x in q_start[b:b + 2])
        if e <= s:
            continue
        node, path = 0, [0]
        while True:
            p = p_all[s + node]
            C, M, gone, went = 0, 1 << 43, [], False
            for child in range(node + 1, e - s) if len(path) < max_kept else ():
                x = int(tokens[s + child])
                if int(parents[s + child]) != node or not 0 <= x < V:
                    continue
                if q_all is not None:
                    q = q_all[s + node]
                    yes = rand(u[s + child]) * q[x] * float(M) < max(p[x] - float(C) / UNIT * q[x], 0.0) * UNIT
                else:
                    r = 0.0 if x in gone else p[x]
                    yes = rand(u[s + child]) * float(M) < r * UNIT
                if yes:
                    node, went = child, True
                    path.append(child)
                    break
                if q_all is not None:
                    C += M
                    M = int(_units(p - float(C) / UNIT * q).sum())
                else:
                    M = max(M - int(_units(np.array([r]))[0]), 0)
                    gone.append(x)
            if went:
                continue
            left = _units(p - float(C) / UNIT * q_all[s + node]) if C else _units(p)
            left[gone] = 0
            if not left.any():
                left = _units(p)
            total = int(left.sum())
            if total:
                t = min(int(np.floor(rand(u_next[b]) * float(total))), total - 1)
                after[b] = int(np.searchsorted(np.cumsum(left), t, side="right"))
            break
        kept[b, :len(path)], n_kept[b] = path, len(path)
    return kept, n_kept, after


def keep_ref(pages, table, q_start, kv, kept, n_kept):
    """pages [n, H, P, d]"""
    out = pages.clone()
    n_pages, _, P, _ = pages.shape

    def place(b, token):
        if not 0 <= token < kv[b] or token // P >= table.shape[1] or not 0 <= table[b, token // P] < n_pages:
            return None
        return int(table[b, token // P]), int(token % P)

    for b in range(len(kv)):
        n = int(q_start[b + 1] - q_start[b])
        base = int(kv[b]) - n
        for j in range(max(0, min(int(n_kept[b]), n, kept.shape[1]))):
            a, c = place(b, base + int(kept[b, j])), place(b, base + j)
            if a and c:
                out[c[0], :, c[1]] = pages[a[0], :, a[1]]
    return out


def trim_ref(kv, n_kept, table, free, count, P, q_start=None):
    """(lens, stack, left, flags)"""
    free, flags, lens = list(free), 0, []
    top = min(max(count, 0), len(free))
    if top != count:
        flags |= 2
    for b in range(len(kv)):
        have = max(int(kv[b]), 0)
        want = int(n_kept[b]) + (0 if q_start is None else have - int(q_start[b + 1] - q_start[b]))
        n = min(max(want, 0), have)
        if n != want or have != kv[b]:
            flags |= 2
        lens.append(n)
        for col in range(-(-n // P), min(-(-have // P), table.shape[1])):
            if table[b, col] < 0:
                continue
            if top < len(free):
                free[top] = int(table[b, col])
                top += 1
            else:
                flags |= 1
    return lens, free, top, flags
