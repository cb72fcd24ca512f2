"""Plain implementations, in 64 bits, of the operators for many texts over one video, and how far a kernel may be off."""
import numpy as np

from paged_reference import values  # noqa: F401


def attention(q, k, v, scale, sees, parts=1):
    """q [rows, d], k, v [keys, d] float64, sees bool [rows, keys] -> (out, lse, tolerance of out, of lse).

    A row's output is rounded to bf16 (half a step, 2^-8 of it).  Before that every probability is carried in one bf16 (2^-8 of each term of the sum of
    w |v|), or, parts 2, in two (2^-16).  Products of bf16 are exact in 32 bits and their sums over d are off by d 2^-24 of the sum of |q k|, which is what a
    logit is off by, and a probability relatively, in the sum and in the normaliser; an exponential by less than 2^-20 with its argument of up to a few
    hundred; sums of n terms, taken 16 at a time, and over pieces, by n / 16 + 400 roundings."""
    if k.shape[0] == 0 or q.shape[0] == 0:
        return np.zeros_like(q), np.full(len(q), -np.inf), np.full_like(q, 1e-30), np.zeros(len(q))
    x = np.where(sees, q @ k.T * scale, -np.inf)
    m = x.max(1, keepdims=True)
    w = np.exp(x - np.where(np.isfinite(m), m, 0))
    total = w.sum(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        lse = (m + np.log(total))[:, 0]
        w = np.where(total > 0, w / total, 0)
    out, spread = w @ v, w @ np.abs(v)
    d = q.shape[1]
    # (a key whose weight is below 2^-200 is off by a factor of e at most, and stays below anything that counts: the size of its logit says nothing)
    off = 2 * (d + 4) * 2.0 ** -24 * scale * np.where(sees, np.abs(q) @ np.abs(k).T, 0)
    assert off.max() < 1
    off = np.where(w >= 2.0 ** -200, off, 0).max(1)
    assert off.max() < 0.02
    sums = (sees.sum(1) / 16 + 400) * 2.0 ** -24
    carried = 2.0 ** -8 if parts == 1 else 2.0 ** -16
    tol = 2.0 ** -8 * np.abs(out) + 1.01 * (carried + 2.0 ** -19 + 2 * off + 2 * sums)[:, None] * spread + 1e-30
    return out, lse, tol, off + 2.0 ** -20 + sums + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0))


def all_heads(q, k, v, scale, sees, parts=1):
    """q [queries, H_q, d], k, v [keys, H_kv, d], sees [queries, keys] -> the same four."""
    out, tol = np.zeros_like(q), np.zeros_like(q)
    lse, tol_lse = (np.zeros(q.shape[:2]) for _ in range(2))
    for h in range(q.shape[1]):
        g = h // (q.shape[1] // k.shape[1])
        out[:, h], lse[:, h], tol[:, h], tol_lse[:, h] = attention(q[:, h], k[:, g], v[:, g], scale, sees, parts)
    return out, lse, tol, tol_lse


def block_sees(kv_len, q_len, masks=None):
    """bool [q_len, kv_len]: the keys that the queries of a block see."""
    j, t = np.arange(kv_len)[None], np.arange(q_len)[:, None]
    before = kv_len - q_len
    if masks is None:
        return j <= before + t
    bits = np.array([[(int(m) >> max(0, int(x) - before)) & 1 if x - before < 64 else 0 for x in range(kv_len)] for m in masks], dtype=bool).reshape(q_len, kv_len)
    return (j < before) | bits


def shared_attention(q, k_pages, v_pages, table, kv_lens, q_lens, scale, masks=None, parts=1, max_kv=None, max_q=None):
    """Attention over pages, request by request: groups have no part in it -> (out, lse, tolerances, rows that are written)."""
    n_pages, ps = k_pages.shape[:2]
    out, tol = np.zeros_like(q), np.zeros_like(q)
    lse, tol_lse = (np.zeros(q.shape[:2]) for _ in range(2))
    written = np.zeros(len(q), dtype=bool)
    at = 0
    for b, (n, ql) in enumerate(zip(kv_lens, q_lens)):
        rows = slice(at, at + ql)
        if 0 < ql <= (max_q or ql) and ql <= n <= (max_kv or table.shape[1] * ps):
            j = np.arange(n)
            page = table[b, j // ps]
            there = (page >= 0) & (page < n_pages)
            k, v = (np.where(there[:, None, None], x[np.where(there, page, 0), j % ps], 0) for x in (k_pages, v_pages))
            sees = block_sees(n, ql, None if masks is None else masks[rows]) & there[None]
            out[rows], lse[rows], tol[rows], tol_lse[rows] = all_heads(q[rows], k, v, scale, sees, parts)
            written[rows] = True
        at += ql
    return out, lse, tol, tol_lse, written


def cross_attention(q, k, v, q_lens, kv_lens, scale, ranges=None, parts=1):
    out, tol = np.zeros_like(q), np.zeros_like(q)
    lse, tol_lse = (np.zeros(q.shape[:2]) for _ in range(2))
    at = first = 0
    for n, states in zip(q_lens, kv_lens):
        rows, keys = slice(at, at + n), slice(first, first + states)
        sees = np.ones((n, states), dtype=bool)
        if ranges is not None:
            j = np.arange(states)[None]
            sees = (j >= ranges[rows, :1]) & (j < ranges[rows, 1:])
        out[rows], lse[rows], tol[rows], tol_lse[rows] = all_heads(q[rows], k[keys], v[keys], scale, sees, parts)
        at, first = at + n, first + states
    return out, lse, tol, tol_lse


def groups(table, kv_lens, q_lens, n_pages, ps, min_tokens):
    """int32 [3, batch], pair after pair."""
    batch, width = table.shape
    whole = [min((n - q) // ps, width) if 0 < q <= n else 0 for n, q in zip(kv_lens, q_lens)]
    common = [0] * (batch + 2)                            # (of b at b; one more behind the last)
    for b in range(1, batch):
        for i in range(min(whole[b - 1], whole[b])):
            if table[b, i] != table[b - 1, i] or not 0 <= table[b, i] < n_pages:
                break
            common[b] += 1
    goes = [b > 0 and common[b] > 0 and common[b] * ps >= min_tokens and 2 * common[b] >= max(common[b - 1], common[b + 1]) for b in range(batch)]
    answer = np.zeros((3, batch), dtype=np.int32)
    for b in range(batch):
        answer[0, b] = answer[0, b - 1] if goes[b] else b
    for f in sorted(set(answer[0].tolist())):
        members = np.flatnonzero(answer[0] == f)
        answer[1, f] = len(members)
        answer[2, members] = min((common[b] for b in members[1:]), default=0) * ps
    return answer
