"""Plain 64-bit statements of the paged calls, and how far a kernel may be from them.

Attention.  With u = 2^-24 (half a step of fp32), for one row of O:
  scores     an fp32 sum of d products in at most 16 steps that follow each other: |error| <= 16 u scale sum_c |q_c k_c|,
             which moves a probability and the sum it is divided by by that much, relative: twice;
  sums       L terms of one sign for the denominator, and the numerator's: roundings of either sign, 8 sqrt(L) u each way;
  exp, log,  the scalings and the division: a few roundings, 2^-21 together;
  16 bits    a probability in two storage-type terms: bf16 loses half a step of a second term that is half a step of the
             first at most, 2^-9 * 2^-9, doubled for the sum being made of the unrounded ones: 2^-16; fp16 no more.
All of them are relative to sum_t p_t |v_t|, channel by channel.  lse has the first two as they are, and the roundings of its
own size: 4 u |lse| + 2^-20.
"""
import numpy as np
import torch

U = 2.0 ** -24


def map_ref(cached, new, table, free, count, P, T):
    """(q_start, kv, table, slots, positions, left, flags) by the header's rules, one request and one token at a time."""
    table = table.copy()
    B, columns = table.shape
    flags = 0
    top = min(max(count, 0), len(free))
    if top != count:
        flags |= 8
    have = top
    starts, kvs, slots, positions = [], [], np.full(T, -1, np.int64), np.full(T, -1, np.int32)
    at = 0
    for b in range(B):
        c, n = int(cached[b]), int(new[b])
        if c < 0 or n < 0:
            flags |= 8
        c, n = max(c, 0), max(n, 0)
        if at + n > T:
            flags |= 4
        if c + min(n, T) > 2 ** 31 - 1:
            flags |= 8
            c = 2 ** 31 - 1 - min(n, T)
        n = min(n, T - at)
        starts.append(at)
        kvs.append(c + n)
        if -(-(c + n) // P) > columns:
            flags |= 2
        for col in range(-(-c // P), min(-(-(c + n) // P), columns)):
            if have > 0:
                have -= 1
                table[b, col] = free[have]
            else:
                flags |= 1
                table[b, col] = -1
        for i in range(n):
            pos = c + i
            positions[at + i] = pos
            if pos // P < columns and table[b, pos // P] >= 0:
                slots[at + i] = int(table[b, pos // P]) * P + pos % P
        at += n
    return np.array(starts + [at]), np.array(kvs), table, slots, positions, have, flags


def write_ref(rows, slots, pages):
    """rows [H, T, d], pages [n, H, P, d]"""
    pages = pages.clone()
    n, _, P, _ = pages.shape
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < n * P:
            pages[s // P, :, s % P] = rows[:, t]
    return pages


def attn_ref(Q, Kp, Vp, table, q_start, kv_lens, causal, scale):
    """(O, lse, tolerance of O, tolerance of lse, rows that are written); Q [Hq, T, d], everything on the CPU"""
    Q64, K64, V64 = (x.double().numpy() for x in (Q, Kp, Vp))
    Hq, T, d = Q64.shape
    n_pages, Hkv, P, _ = K64.shape
    table, q_start, kv_lens = (np.asarray(x, dtype=np.int64) for x in (table, q_start, kv_lens))
    two_terms = 2.0 ** -16 if Q.dtype != torch.float32 else 0.0
    O, lse = np.zeros((Hq, T, d)), np.full((Hq, T), -np.inf)
    tol_o, tol_l = np.zeros((Hq, T, d)), np.zeros((Hq, T))
    written = np.zeros(T, bool)
    for b in range(table.shape[0]):
        s, e = int(q_start[b]), int(q_start[b + 1])
        n, kv = e - s, max(int(kv_lens[b]), 0)
        if n <= 0:
            continue
        written[s:e] = True
        key = np.arange(min(kv, table.shape[1] * P))
        ids = table[b][key // P]
        there = (ids >= 0) & (ids < n_pages)
        key, ids = key[there], ids[there]
        for h in range(Hq):
            K, V = K64[ids, h // (Hq // Hkv), key % P], V64[ids, h // (Hq // Hkv), key % P]
            for i in range(n):
                sees = key <= kv - n + i if causal else np.ones(len(key), bool)
                if not sees.any():
                    continue
                k, v, q = K[sees], V[sees], Q64[h, s + i]
                with np.errstate(invalid="ignore"):
                    x = (k @ q) * scale
                    m = x.max()
                    p = np.exp(x - m)
                    total = p.sum()
                    O[h, s + i] = p @ v / total
                    lse[h, s + i] = m + np.log(total)
                    off = 16 * U * scale * (np.abs(k) @ np.abs(q)).max() + 8 * U * np.sqrt(len(k))
                    tol_o[h, s + i] = (2 * off + 2.0 ** -21 + two_terms) * (p @ np.abs(v) / total)
                    tol_l[h, s + i] = off + 4 * U * abs(lse[h, s + i]) + 2.0 ** -20
    return O, lse, tol_o, tol_l, written


def check_attn(O, lse, ref, fill, what=""):
    """Written rows within the tolerances (not-a-number and infinite where the reference is), the others as they were."""
    r_o, r_l, t_o, t_l, written = ref
    O, lse = O[0].double().cpu().numpy(), lse[0].double().cpu().numpy()
    assert (O[:, ~written] == fill).all() and (lse[:, ~written] == fill).all(), f"{what}: rows of no request were written"
    for name, x, y, tol in (("O", O[:, written], r_o[:, written], t_o[:, written]), ("lse", lse[:, written], r_l[:, written], t_l[:, written])):
        fin = np.isfinite(y)
        assert np.array_equal(np.isfinite(x), fin), f"{what}: {name} is finite where it should not be, or the other way round"
        assert np.array_equal(x[np.isinf(y)], y[np.isinf(y)]), f"{what}: {name}'s infinities"
        worst = np.max(np.abs(x[fin] - y[fin]) - tol[fin], initial=-1.0)
        assert worst <= 0, f"{what}: {name} is beyond its tolerance by {worst:.3e}"
