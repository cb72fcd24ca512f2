"""Plain implementations of the paged operators, in 64 bits and in Python's loops, and how far a kernel may be off."""
import numpy as np


def values(bits):
    """bf16 bit patterns -> float64."""
    return (np.asarray(bits).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def visible(kv_len, q_len, t, window=0, n_sinks=0, mask=None):
    """The keys that query t of the block sees, by the definition."""
    before, p = kv_len - q_len, kv_len - q_len + t
    out = []
    for j in range(kv_len):
        if j >= before and not (j <= p if mask is None else (int(mask) >> (j - before)) & 1):
            continue
        if window and not (j > p - window or j < n_sinks):
            continue
        out.append(j)
    return np.array(out, dtype=np.int64)


def attention(q, k, v, scale, sees):
    """q [rows, d], k, v [keys, d] float64, sees: a list of key indices a row -> (out, lse, tolerance of out, of lse).

    A row's output is rounded to bf16 (half a step, 2^-8 of it).  Before that every probability is carried in two bf16 (2^-16 of each term of
    the sum of w |v|).  Products of bf16 are exact in 32 bits and their sums over d are off by d 2^-24 of the sum of |q k|, which is what a
    logit is off by, and a probability relatively, in the sum and in the normaliser; an exponential by less than 2^-20 with its argument of up
    to a few hundred, sums of n terms taken eight at a time and more by n / 8 + 64 roundings."""
    out, lse = np.zeros_like(q), np.full(len(q), -np.inf)
    tol, tol_lse = np.full_like(q, 1e-30), np.zeros(len(q))
    d = q.shape[1]
    for i, js in enumerate(sees):
        if len(js) == 0:
            continue
        x = k[js] @ q[i] * scale
        m = x.max()
        w = np.exp(x - m)
        lse[i] = m + np.log(w.sum())
        w /= w.sum()
        out[i] = w @ v[js]
        off = 2 * (d + 4) * 2.0 ** -24 * scale * (np.abs(k[js]) @ np.abs(q[i])).max()
        assert off < 0.02
        spread = w @ np.abs(v[js])
        sums = (len(js) / 8 + 64) * 2.0 ** -24
        tol[i] = 2.0 ** -8 * np.abs(out[i]) + 1.01 * (2.0 ** -16 + 2.0 ** -19 + 2 * off + 2 * sums) * spread + 1e-30
        tol_lse[i] = off + 2.0 ** -20 + sums + 2.0 ** -22 * abs(lse[i])
    return out, lse, tol, tol_lse


def paged_attention(q, k_pages, v_pages, table, kv_lens, q_lens, scale, window=0, n_sinks=0, masks=None, max_kv=None, max_q=64):
    """q [tokens, H_q, d], pools [pages, page_size, H_kv, d] float64 -> (out, lse, tolerances, rows that are written)."""
    n_pages, ps, hkv, d = k_pages.shape
    tokens, hq, _ = q.shape
    out, tol = np.zeros_like(q), np.zeros_like(q)
    lse, tol_lse = np.zeros((tokens, hq)), np.zeros((tokens, hq))
    written = np.zeros(tokens, dtype=bool)
    at = 0
    for b, (n, ql) in enumerate(zip(kv_lens, q_lens)):
        if 0 < ql <= max_q and ql <= n <= (table.shape[1] * ps if max_kv is None else max_kv):
            sees = []
            for t in range(ql):
                js = visible(n, ql, t, window, n_sinks, None if masks is None else masks[at + t])
                sees.append(js[[0 <= table[b][j // ps] < n_pages for j in js]] if len(js) else js)
            used = sorted(set(int(j) for js in sees for j in js))
            place = {j: i for i, j in enumerate(used)}
            k = np.array([k_pages[table[b][j // ps], j % ps] for j in used]).reshape(len(used), hkv, d)
            v = np.array([v_pages[table[b][j // ps], j % ps] for j in used]).reshape(len(used), hkv, d)
            sees = [np.array([place[int(j)] for j in js], dtype=np.int64) for js in sees]
            for h in range(hq):
                g = h // (hq // hkv)
                o = attention(q[at:at + ql, h], k[:, g], v[:, g], scale, sees)
                out[at:at + ql, h], lse[at:at + ql, h], tol[at:at + ql, h], tol_lse[at:at + ql, h] = o
            written[at:at + ql] = True
        at += ql
    return out, lse, tol, tol_lse, written


def frequencies(rot, base, kind=None, factor=1.0, original_len=0.0, fast=32.0, slow=1.0):
    """Radians a position of every pair, in extended precision."""
    i = np.arange(rot // 2, dtype=np.longdouble)
    base = np.longdouble(base)
    if kind == "base":
        base = base * np.longdouble(factor) ** (np.longdouble(rot) / (rot - 2))
    f = base ** (-2 * i / rot)
    if kind == "linear":
        f = f / factor
    if kind == "by-parts":
        turns = original_len * f / (2 * np.longdouble("3.14159265358979323846264338327950288"))
        keep = np.clip((turns - slow) / (fast - slow), 0, 1)
        f = f * keep + f / factor * (1 - keep)
    return f


def rope(x, positions, freq, interleaved, magnitude):
    """x [tokens, heads, d] float64 -> (turned, tolerance): the angles modulo a turn in extended precision.

    Rounding to bf16 is half a step; the angle's upper 32 bits as fp32, the sine and cosine and two fp32 products and a sum are
    off by less than 2^-20 of |a| + |b|."""
    rot = 2 * len(freq)
    pi2 = 2 * np.longdouble("3.14159265358979323846264338327950288")
    angle = np.fmod(np.outer(np.asarray(positions, dtype=np.longdouble), freq), pi2)
    c, s = (np.asarray(f(angle), dtype=np.float64)[:, None] * magnitude for f in (np.cos, np.sin))
    y, tol = x.copy(), np.zeros_like(x)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size = (np.abs(x[..., a]) + np.abs(x[..., b])) * abs(magnitude) * 2.0 ** -20
    tol[..., a], tol[..., b] = size, size
    tol[..., :rot] += 2.0 ** -8 * np.abs(y[..., :rot])
    return y, tol


def assign(old, parent, keep, new, n_pages, ps, width, window=0, n_sinks=0):
    """-> (table, copy_start, copy_rows, ref_counts, status), request by request."""
    batch = len(parent)
    table = np.full((batch, width), -1, dtype=np.int32)
    start, rows, status = (np.zeros(batch, dtype=np.int32) for _ in range(3))
    refs = np.zeros(n_pages, dtype=np.int32)
    kept, valid = [], []
    for b in range(batch):
        p, k, n = int(parent[b]), int(keep[b]), int(new[b])
        ok = -1 <= p < len(old) and 0 <= k <= n and (k == 0 or p >= 0)
        ok = ok and -(-k // ps) <= old.shape[1] and -(-n // ps) <= width
        valid.append(ok)
        pages = []
        for i in range(-(-k // ps) if ok else 0):
            page = int(old[p, i])
            if not 0 <= page < n_pages:
                page = -1
            if window and all(j >= n_sinks and not j > k - window for j in (i * ps, i * ps + ps - 1)):
                page = -1
            pages.append(page)
        kept.append(pages)
    whole = {p for b in range(batch) for p in kept[b][:int(keep[b]) // ps] if valid[b]}
    taken, needs = set(), []
    for b in range(batch):
        leaves = False
        if valid[b] and int(keep[b]) % ps:
            page = kept[b][-1]
            leaves = page >= 0 and (page in whole or page in taken)
            taken.add(page)
            if leaves:
                kept[b][-1] = -1
            needs.append((-(-int(new[b]) // ps) - len(kept[b]) + (kept[b][-1] < 0), leaves))
        else:
            needs.append((-(-int(new[b]) // ps) - len(kept[b]) if valid[b] else 0, False))
        for page in kept[b]:
            if page >= 0:
                refs[page] += 1
    free = [p for p in range(n_pages) if refs[p] == 0]
    at = 0
    for b in range(batch):
        need, leaves = needs[b]
        table[b, :len(kept[b])] = kept[b]
        status[b] = 0 if valid[b] else -1
        if need and at + need > len(free):
            status[b] = -5
        elif need:
            end = -(-int(new[b]) // ps)
            table[b, end - need:end] = free[at:at + need]
            for page in free[at:at + need]:
                refs[page] = 1
            if leaves:
                start[b], rows[b] = int(keep[b]) // ps * ps, int(keep[b]) % ps
        at += need
    return table, start, rows, refs, status
