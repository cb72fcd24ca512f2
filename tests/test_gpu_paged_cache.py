"""specvlm_rope_append, specvlm_pages_assign and specvlm_pages_copy against plain implementations, and a run of the paged
operators together, as a serving loop makes their calls."""
import numpy as np
import pytest
import torch

import oracle
import paged_reference as R
from gpu_util import dev_bf16, host_bits, host_f64, rnd_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2508_16201_amd import binding
    binding.lib()
    return binding


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def tables(seed, lens, ps, spare=2, pad=1):
    """Pages in no order for requests of these lengths."""
    rng = np.random.default_rng(seed)
    counts = [-(-max(n, 0) // ps) for n in lens]
    ids, at = rng.permutation(sum(counts) + spare), 0
    table = np.full((len(lens), max(counts) + pad), -1, dtype=np.int32)
    for b, c in enumerate(counts):
        table[b, :c] = ids[at:at + c]
        at += c
    return table, sum(counts) + spare


# ------------------------------------------------------------------------------------------------------------- rope
def check_rope(B, seed, kv_lens, q_lens, heads, ps, rot, *, interleaved=False, magnitude=1.0, positions=None, behind=0, ragged=True, head_major=False,
               table=None, with_q=True, with_k=True, in_place=False, **scaling):
    hq, hkv, d = heads
    n = sum(q_lens) + behind
    made, total = tables(seed, kv_lens, ps)
    table = made if table is None else table(made, total)
    q, k, v = (rnd_bits((n, h, d), (seed, h, i)) for i, h in enumerate((hq, hkv, hkv)))
    pools = [rnd_bits((total, ps, hkv, d), (seed, 5 + i)) for i in range(2)]
    on = [dev_bf16(np.ascontiguousarray(p.transpose(0, 2, 1, 3))).transpose(1, 2) if head_major else dev_bf16(p) for p in pools]
    base = scaling.pop("base", 1e6)
    turns = B.rope_turns(rot, base, **scaling) if rot else None
    qd = dev_bf16(q) if with_q else None
    out = None if not with_q else qd if in_place else torch.full_like(qd, 7.0)
    got = B.rope_append(*((dev_bf16(k), dev_bf16(v), *on, i32(table)) if with_k else (None,) * 5), i32(kv_lens), q=qd, q_out=out, turns=turns,
                        interleaved=interleaved, magnitude=magnitude, positions=None if positions is None else i32(positions),
                        cu_q=i32(np.concatenate([[0], np.cumsum(q_lens)])) if ragged else None)
    torch.cuda.synchronize()
    f = R.frequencies(rot, base, scaling.get("scaling"), scaling.get("factor", 1.0), scaling.get("original_len", 0.0)) if rot else np.zeros(0, dtype=np.longdouble)
    place, request = np.full(n, -1, dtype=np.int64), np.full(n, -1, dtype=np.int64)
    at = 0
    for b, (m, ql) in enumerate(zip(kv_lens, q_lens)):
        if m >= ql:
            place[at:at + ql], request[at:at + ql] = np.arange(m - ql, m), b
        at += ql
    live = place >= 0
    pos = place if positions is None else np.asarray(positions)
    if with_q:
        want, tol = R.rope(R.values(q), pos, f, interleaved, magnitude)
        have = host_f64(got)
        assert (np.abs(have - want)[live] <= tol[live]).all(), (np.abs(have - want)[live] - tol[live]).max()
        assert (have[~live] == (R.values(q)[~live] if in_place else 7.0)).all()
    want = [R.values(p) for p in pools]
    tol = np.zeros_like(want[0])
    if with_k:
        turned, off = R.rope(R.values(k), pos, f, interleaved, magnitude)
        for t in np.flatnonzero(live):
            column = place[t] // ps
            page = table[request[t], column] if column < table.shape[1] else -1
            if 0 <= page < total:
                want[0][page, place[t] % ps], tol[page, place[t] % ps] = turned[t], off[t]
                want[1][page, place[t] % ps] = R.values(v)[t]
    assert (np.abs(host_f64(on[0]) - want[0]) <= tol).all()
    assert np.array_equal(host_f64(on[1]), want[1])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,rot", [((4, 1, 64), 64), ((14, 2, 64), 16), ((28, 4, 128), 128), ((64, 8, 128), 64), ((5, 5, 128), 32), ((3, 3, 64), 0), ((1, 1, 128), 112)])
def test_rope_shapes(B, heads, rot, interleaved):
    check_rope(B, rot + 1, [100, 7, 33, 1], [6, 7, 1, 1], heads, 16, rot, interleaved=interleaved)


@pytest.mark.parametrize("kind", [dict(scaling="linear", factor=8.0), dict(scaling="base", factor=4.0, base=1e4),
                                  dict(scaling="by-parts", factor=32.0, original_len=4096, magnitude=1.35), dict(magnitude=0.0), dict(magnitude=-2.0)])
def test_rope_scalings_at_far_positions(B, kind):
    check_rope(B, 3, [50, 20], [9, 20], (8, 2, 128), 32, 128, positions=np.random.default_rng(1).integers(0, 2 ** 31 - 1, 29), **kind)


def test_rope_positions_of_every_size(B):
    """0, 1, the largest and smallest ints, and neighbours of powers of two."""
    at = [0, 1, 2 ** 31 - 1, -2 ** 31, -1] + [2 ** i + j for i in range(4, 31, 3) for j in (-1, 0, 1)]
    for interleaved in (False, True):
        check_rope(B, 4, [64], [len(at)], (4, 2, 64), 16, 64, positions=at, interleaved=interleaved, base=1e4)


def test_rope_ragged_and_padded(B):
    """Empty requests, one with fewer cached tokens than new ones, and tokens behind the last request."""
    check_rope(B, 5, [30, 0, 3, 16, 64], [4, 0, 5, 16, 1], (14, 2, 64), 16, 64, behind=5)
    check_rope(B, 6, [30, 1, 16], [2, 2, 2], (14, 2, 64), 16, 64, ragged=False)
    check_rope(B, 6, [30, 1, 16], [2, 2, 2], (14, 2, 64), 16, 64, behind=2, in_place=True)
    lens = [int(n) for n in np.random.default_rng(2).integers(1, 90, 150)]
    check_rope(B, 7, lens, [min(n, 1 + i % 3) for i, n in enumerate(lens)], (4, 2, 64), 16, 32)


def test_rope_pages_that_are_none(B):
    """Rows of missing pages are dropped, and nothing else changes."""
    def broken(table, total):
        table[0, 2], table[1, 0] = -1, total
        return table[:, :4]                               # (the table ends before the third request's tokens do)
    check_rope(B, 8, [60, 10, 70], [40, 10, 20], (8, 2, 128), 16, 128, table=broken)


@pytest.mark.parametrize("ps,head_major", [(16, True), (48, False), (256, True)])
def test_rope_pages(B, ps, head_major):
    check_rope(B, 9, [500, 77], [77, 77], (14, 2, 64), ps, 32, head_major=head_major)


def test_rope_of_queries_or_keys_alone(B):
    check_rope(B, 10, [40, 9], [3, 9], (8, 2, 128), 16, 64, with_q=False)
    check_rope(B, 11, [40, 9], [3, 9], (8, 2, 128), 16, 64, with_k=False)
    check_rope(B, 12, [40, 9], [3, 9], (8, 2, 128), 16, 64, with_k=False, in_place=True)
    q = rnd_bits((6, 4, 64), 13)
    got = B.rope_append(None, None, None, None, None, None, q=dev_bf16(q), turns=B.rope_turns(64, 1e4), positions=i32(range(6)))
    want, tol = R.rope(R.values(q), np.arange(6), R.frequencies(64, 1e4), False, 1.0)
    assert (np.abs(host_f64(got) - want) <= tol).all()


def test_rope_of_a_long_prompt(B):
    """More tokens than the waves that fill the chip."""
    check_rope(B, 14, [2100, 1700], [2100, 1600], (28, 4, 128), 16, 128, interleaved=True)


def test_rope_of_a_prompt_that_is_not_kept_near(B):
    n = 3400
    assert n * (64 + 2 * 8) * 128 * 4 >= 128 << 20
    check_rope(B, 15, [n + 100], [n], (64, 8, 128), 64, 96)


def test_rope_strides(B):
    n, hq, hkv, d, ps = 5, 6, 2, 64, 16
    fused = rnd_bits((n, hq + 2 * hkv, d), 15)                           # q, k and v of a token side by side, as one projection leaves them
    one = dev_bf16(fused)
    pool = torch.zeros((2, 3, 8, ps, d), dtype=torch.bfloat16, device="cuda")
    k_pages, v_pages = pool[0, :, 1:5:2].transpose(1, 2), pool[1, :, 1:5:2].transpose(1, 2)
    turns = B.rope_turns(d, 1e4)
    out = B.rope_append(one[:, hq:hq + hkv], one[:, hq + hkv:], k_pages, v_pages, i32([[2, 0]]), i32([20]), q=one[:, :hq],
                        q_out=torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda"), turns=turns)
    x, tol = R.rope(R.values(fused), np.arange(15, 20), R.frequencies(d, 1e4), False, 1.0)
    assert (np.abs(host_f64(out) - x[:, :hq]) <= tol[:, :hq]).all()
    for t, j in enumerate(range(15, 20)):
        page = [2, 0][j // ps]
        assert (np.abs(host_f64(k_pages[page, j % ps]) - x[t, hq:hq + hkv]) <= tol[t, hq:hq + hkv]).all()
        assert np.array_equal(host_bits(v_pages[page, j % ps]), fused[t, hq + hkv:])
    assert (pool[:, :, 0::2] == 0).all() and (pool[:, :, 5:] == 0).all()


# ----------------------------------------------------------------------------------------------------------- assign
def check_assign(B, old, parent, keep, new, n_pages, ps, width=None, window=0, n_sinks=0, **kw):
    width = old.shape[1] if width is None else width
    got = B.pages_assign(i32(old), i32(parent), i32(keep), i32(new), n_pages, ps, max_pages=width, window=window, n_sinks=n_sinks, **kw)
    want = R.assign(old, parent, keep, new, n_pages, ps, width, window, n_sinks)
    for name, g, w in zip(("table", "copy_start", "copy_rows", "ref_counts", "status"), got, want):
        assert np.array_equal(g.cpu().numpy(), w), name
    return want


def test_assign_by_hand(B):
    """Three rows of which two go on from one: whole pages shared, the last page with the first, a copy for the second."""
    old = np.array([[4, 2, 7, -1], [0, 5, -1, -1]], dtype=np.int32)
    table, start, rows, refs, status = check_assign(B, old, [0, 0, -1], [40, 40, 0], [41, 60, 17], 10, 16)
    assert table.tolist() == [[4, 2, 7, -1], [4, 2, 0, 1], [3, 5, -1, -1]]
    assert start.tolist() == [0, 32, 0] and rows.tolist() == [0, 8, 0]
    assert refs.tolist() == [1, 1, 2, 1, 2, 1, 0, 1, 0, 0] and status.tolist() == [0, 0, 0]


def test_assign_a_page_that_another_keeps_whole(B):
    """A row goes back into the middle of a page that its sibling keeps: the sibling's tokens stay as they are."""
    old = np.array([[3, 1]], dtype=np.int32)
    table, start, rows, _, _ = check_assign(B, old, [0, 0, 0], [10, 32, 10], [12, 32, 40], 6, 16, width=3)
    assert table.tolist() == [[0, -1, -1], [3, 1, -1], [2, 4, 5]] and rows.tolist() == [10, 0, 10]


def test_assign_ends_frees_and_runs_out(B):
    old = np.array([[0, 1, 2], [3, 4, -1], [5, -1, -1]], dtype=np.int32)
    table, _, _, refs, status = check_assign(B, old, [0, 1, 2], [0, 20, 16], [0, 90, 17], 7, 16, width=6)
    assert status.tolist() == [0, 0, -5] and (refs == 1).sum() == 7
    check_assign(B, old, [0, 0, 1, 2], [40, 40, 20, 0], [48, 49, 20, 16], 6, 16)
    check_assign(B, old, [0, 1, 2], [48, 32, 16], [48, 32, 16], 6, 16)


def test_assign_rows_that_do_not_fit_together(B):
    old = np.array([[0, 1, 2], [3, 4, -1]], dtype=np.int32)
    _, _, _, _, status = check_assign(B, old, [2, -2, 0, 0, -1, 0, 1, 1, 1, 0], [4, 4, -1, 9, 3, 49, 20, 20, 20, 48], [5, 5, 3, 8, 4, 60, 49, 33, 48, 48], 12, 16)
    assert status.tolist() == [-1, -1, -1, -1, -1, -1, -1, 0, 0, 0]
    check_assign(B, old, [0, 1], [2 ** 31 - 1, 5], [2 ** 31 - 1, 2 ** 31 - 1], 12, 16)


def test_assign_keeps_pages_that_are_none(B):
    old = np.array([[7, -1, 99, 2], [2 ** 31 - 1, 3, -5, -1]], dtype=np.int32)
    check_assign(B, old, [0, 1, 1], [60, 33, 40], [64, 50, 41], 8, 16)


@pytest.mark.parametrize("window,n_sinks", [(1, 0), (16, 4), (20, 17), (100, 16), (2 ** 31 - 1, 0), (5, 2 ** 31 - 1)])
def test_assign_gives_up_what_a_window_hides(B, window, n_sinks):
    rng = np.random.default_rng(window % 97)
    old, total = tables(3, [500, 130, 64, 16], 16)
    keep = np.array([500, 100, 64, 16, 31, 499])
    check_assign(B, old, [0, 1, 2, 3, 0, 0], keep, keep + rng.integers(0, 9, 6), total + 5, 16, width=40, window=window, n_sinks=n_sinks)


@pytest.mark.parametrize("seed", range(20))
def test_assign_random(B, seed):
    rng = np.random.default_rng(seed)
    batch, rows = int(rng.choice([1, 3, 30, 300, 1500])), int(rng.choice([1, 7, 200]))
    ps = int(rng.choice([16, 48, 128]))
    longest = int(rng.choice([30, 700, 9000])) if batch < 1500 else 300
    lens = rng.integers(0, longest + 1, rows)
    old, total = tables(seed, lens, ps, pad=2)
    parent = rng.integers(-1, rows, batch)
    keep = np.where(parent >= 0, (lens[parent] * rng.choice([1.0, 1.0, 0.5, 0.0], batch)).astype(int), 0)
    new = keep + rng.integers(0, 3 * ps, batch)
    new[rng.random(batch) < 0.1] = 0
    keep = np.minimum(keep, new)
    used = sum(R.assign(old, parent, keep, new, total + batch * 5, ps, old.shape[1] + 4)[3] > 0)
    n_pages = max(int(old.max()) + 1, int(used * rng.choice([0.7, 1.0, 1.3])))           # too few, just enough, plenty
    check_assign(B, old, parent, keep, new, n_pages, ps, width=old.shape[1] + 4)


def test_assign_empty_pools_and_tables(B):
    old = np.zeros((2, 0), dtype=np.int32)
    check_assign(B, old, [0, -1], [0, 0], [0, 0], 0, 16)
    check_assign(B, old, [0, -1], [0, 0], [5, 17], 0, 16, width=3)
    check_assign(B, old, [-1, 1], [0, 0], [5, 17], 3, 16, width=3)
    check_assign(B, np.array([[0]], dtype=np.int32), [0], [16], [16], 1, 16)


def test_assign_replayed_while_the_lengths_change(B):
    """Captured once, ping-pong between two tables, with eager work between the replays."""
    ps, n_pages, width = 16, 64, 20
    first, second = torch.full((4, width), -1, dtype=torch.int32, device="cuda"), torch.zeros((4, width), dtype=torch.int32, device="cuda")
    parent, keep, new = i32([0, 1, 2, 3]), i32([0] * 4), i32([1] * 4)
    ws = B.new_workspace(B.lib().specvlm_pages_assign_workspace_bytes(4, n_pages))
    call = lambda: B.pages_assign(first, parent, keep, new, n_pages, ps, out=second, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    host, rng, length = np.full((4, width), -1, dtype=np.int32), np.random.default_rng(0), np.zeros(4, dtype=int)
    for step in range(6):
        p = rng.integers(0, 4, 4) if step else np.arange(4)
        k = (length[p] * rng.choice([1, 1, 0.6], 4)).astype(int)
        n = k + rng.integers(0, 30, 4)
        for t, x in ((first, host), (parent, p), (keep, k), (new, n)):
            t.copy_(i32(x))
        ws.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        want = R.assign(host, p, k, n, n_pages, ps, width)
        for g, w in zip(got, want):
            assert np.array_equal(g.cpu().numpy(), w), step
        host, length = want[0], n


# ------------------------------------------------------------------------------------------------------------- copy
def check_copy(B, seed, layers, heads, src_lens, dst_lens, src_ps, dst_ps, n_rows, src_start, dst_start, *, src_row=None, idx=None, cut=False, max_rows=None,
               one_pool=False, with_v=True, head_major=False, break_tables=None):
    hkv, d = heads
    src_table, src_total = tables(seed, src_lens, src_ps)
    dst_table, dst_total = (src_table, src_total) if one_pool else tables(seed + 1, dst_lens, dst_ps)
    if break_tables:
        src_table, dst_table = break_tables(src_table.copy(), src_total, dst_table.copy(), dst_total)
    src = [rnd_bits((layers, src_total, src_ps, hkv, d), (seed, i)) for i in range(2)]
    dst = src if one_pool else [rnd_bits((layers, dst_total, dst_ps, hkv, d), (seed, 2 + i)) for i in range(2)]
    def up(p):
        return dev_bf16(np.ascontiguousarray(p.transpose(0, 1, 3, 2, 4))).transpose(2, 3) if head_major else dev_bf16(p)
    on_src = [up(p) for p in src]
    on_dst = on_src if one_pool else [up(p) for p in dst]
    batch = len(dst_table)
    more = {}
    if idx is not None:
        if cut:
            more = {"row_idx": i32(np.concatenate(idx) if sum(map(len, idx)) else np.zeros(1)), "cu_idx": i32(np.concatenate([[0], np.cumsum([len(x) for x in idx])]))}
        else:
            width = max(max(len(x) for x in idx), 1)
            more = {"row_idx": i32([list(x) + [-1] * (width - len(x)) for x in idx])}
            max_rows = width if max_rows is None else max_rows
    counts = [len(x) for x in idx] if n_rows is None else n_rows
    max_rows = max(max(counts), 1) if max_rows is None else max_rows
    B.pages_copy(on_src[0], on_src[1] if with_v else None, i32(src_table), on_dst[0], on_dst[1] if with_v else None, i32(dst_table),
                 None if n_rows is None else i32(n_rows), max_rows, src_row=None if src_row is None else i32(src_row),
                 src_start=None if src_start is None else i32(src_start), dst_start=None if dst_start is None else i32(dst_start), **more)
    torch.cuda.synchronize()
    want = [p.copy() for p in dst]
    for b in range(batch):
        row = b if src_row is None else src_row[b]
        for i in range(max(0, min(counts[b], max_rows))):
            s = (src_start[b] if src_start else 0) + (idx[b][i] if idx is not None else i)
            t = (dst_start[b] if dst_start else 0) + i
            at = [-1, -1]
            for side, (table, token, r, ps, total) in enumerate(((src_table, s, row, src_ps, src_total), (dst_table, t, b, dst_ps, dst_total))):
                if 0 <= r < len(table) and 0 <= token < table.shape[1] * ps and 0 <= table[r, token // ps] < total:
                    at[side] = table[r, token // ps]
            if at[1] >= 0:
                for w, p in zip(want[:2 if with_v else 1], src):
                    w[:, at[1], t % dst_ps] = p[:, at[0], s % src_ps] if at[0] >= 0 else 0
    for g, w in zip(on_dst, want):
        assert np.array_equal(host_bits(g), w)


HEADS = [(1, 64), (2, 64), (4, 128), (8, 128), (24, 128), (3, 64)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("head_major", [False, True])
def test_copy_lists_into_another_pool(B, heads, head_major):
    """The pruned cache of each request, into pages of another size, after a prefix."""
    rng = np.random.default_rng(1)
    idx = [np.sort(rng.choice(n, m, replace=False)) for n, m in ((300, 31), (50, 50), (7, 1), (90, 0))]
    args = (B, 1, 3, heads, [300, 60, 20, 100], [40, 60, 20, 5], 16, 48)
    for cut in (False, True):
        check_copy(*args, None if cut else [31, 50, 1, 0], [0, 5, 9, 0], [3, 0, 19, 0], idx=idx, cut=cut, head_major=head_major)


@pytest.mark.parametrize("heads", HEADS)
def test_copy_accepted_nodes_in_place(B, heads):
    """Rows that lie in each other's way, in one page and over pages, more of them than a workgroup holds at once."""
    rng = np.random.default_rng(2)
    lens = [100, 33, 16, 700]
    idx = [[1, 3, 4, 9], [1, 2, 3], [], np.sort(rng.choice(np.arange(1, 600), 200, replace=False))]
    check_copy(B, 2, 2, heads, lens, None, 16, 16, [4, 3, 0, 200], [80, 16, 3, 90], [81, 17, 4, 91], idx=idx, one_pool=True)
    check_copy(B, 3, 2, heads, lens, None, 16, 16, [50, 10, 1, 599], [30, 20, 9, 101], [3, 11, 8, 100], one_pool=True)


def test_copy_a_forks_page(B):
    check_copy(B, 4, 4, (4, 128), [100, 40], [100, 40, 60], 32, 32, [4, 8, 31], [96, 32, 64], [96, 32, 32], src_row=[0, 1, 0])


def test_copy_counts_and_rows_that_are_off(B):
    """Counts beyond the list's room and below 0, parents that are no rows, tokens outside the tables, pages that are none."""
    def broken(s, s_total, t, t_total):
        s[0, 1], t[1, 0] = -1, t_total
        return s, t
    check_copy(B, 5, 2, (2, 64), [64, 64], [64, 64, 64, 64], 16, 16, [40, 20, -3, 2], [0, 60, 0, 0], [10, 5, 0, 50], src_row=[0, 1, 0, 2], max_rows=30, break_tables=broken)
    check_copy(B, 6, 2, (2, 64), [64, 64], [64, 64], 16, 16, [3, 3], [0, 0], [0, 0], idx=[[-5, 70, 3], [2 ** 31 - 1, 63, 64]], max_rows=3)
    check_copy(B, 7, 2, (2, 64), [64, 64], [64, 64], 16, 16, [3, 3], [2 ** 31 - 1, -2], [-1, 2 ** 31 - 2])


def test_copy_that_is_not_kept_near(B):
    idx = [np.arange(0, 1000)[np.random.default_rng(3).random(1000) < 0.9]]
    assert 2 * 2 * 8 * 128 * 20 * len(idx[0]) >= 64 << 20
    check_copy(B, 9, 20, (8, 128), [1000], [1000], 16, 64, [len(idx[0])], None, [7], idx=idx)


def test_copy_keys_alone_without_starts(B):
    check_copy(B, 8, 2, (4, 128), [64, 30], [64, 30], 16, 32, [64, 30], None, None, with_v=False)


def test_copy_pools_beyond_32_bits(B):
    """Layers whose elements lie past 2^32."""
    layers, pages, ps, h, d = 3, 1 << 16, 32, 8, 128                     # 2^31 elements a layer
    k = torch.zeros((layers, pages + 1, ps, h, d), dtype=torch.bfloat16, device="cuda")
    assert k.stride(0) > 2 ** 31 and k.stride(0) * 2 > 2 ** 32
    mark = torch.randn((layers, 5, h, d), device="cuda").to(torch.bfloat16)
    k[:, pages, 3:8] = mark
    k[:, 7, 3:8] = 1.0
    B.pages_copy(k, None, i32([[pages]]), k, None, i32([[7]]), i32([5]), 5, src_start=i32([3]), dst_start=i32([20]))
    assert torch.equal(k[:, 7, 20:25], mark) and (k[:, 7, 3:8] == 1).all()


def test_binding_refusals(B):
    k = torch.zeros((2, 4, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
    t, one = i32([[0, 1]]), i32([1])
    new = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    bad = [
        lambda: B.paged_attn(q.float(), k[0], k[1], t, one, 0.1), lambda: B.paged_attn(q, k[0].float(), k[1].float(), t, one, 0.1),
        lambda: B.paged_attn(q, k[0], k[1], t.long(), one, 0.1), lambda: B.paged_attn(q, k[0], k[1], t, one.long(), 0.1),
        lambda: B.paged_attn(q, k[0], k[1, :3], t, one, 0.1), lambda: B.paged_attn(q, k[0], k[1], t, i32([1, 1]), 0.1),
        lambda: B.paged_attn(q, k[0], k[1], t, one, 0.1, cu_q=i32([0, 1])), lambda: B.paged_attn(q, k[0], k[1], t, one, 0.1, cu_q=i32([0]), max_q_len=1),
        lambda: B.paged_attn(q[..., :32], k[0], k[1], t, one, 0.1), lambda: B.paged_attn(q.expand(3, 4, 64), k[0], k[1], i32([[0, 1]] * 2), i32([1, 1]), 0.1),
        lambda: B.paged_attn(q, k[0], k[1], t, one, 0.1, out=torch.zeros_like(q).float()),
        lambda: B.paged_attn(q, k[0], k[1], t, one, 0.1, out=torch.zeros((1, 4, 128), dtype=torch.bfloat16, device="cuda")[..., ::2]),
        lambda: B.paged_attn(q, k[0], k[1], t, one, 0.1, ancestor_mask=i32([1])), lambda: B.paged_attn(q, k[0], k[1], t, one.cpu(), 0.1),
        lambda: B.rope_append(new, None, k[0], k[1], t, one), lambda: B.rope_append(new, new, k[0], k[1], t, one, q=q[..., :32]),
        lambda: B.rope_append(new, new, k[0], k[1], t, one, positions=i32([1, 2])), lambda: B.rope_append(new, new, k[0], k[1], i32([[0], [1]]), one),
        lambda: B.rope_append(None, None, None, None, None, one), lambda: B.rope_append(new, new, k[0], k[1], t, one, turns=torch.zeros(4, device="cuda")),
        lambda: B.rope_append(new, new, None, None, t, one), lambda: B.rope_append(new, new, k[0], k[1], t, None),
        lambda: B.rope_append(new.expand(1, 2, 64).float(), new, k[0], k[1], t, one),
        lambda: B.pages_assign(t, one, one, i32([1, 2]), 4, 16), lambda: B.pages_assign(t, one, one, one.long(), 4, 16), lambda: B.pages_assign(t, one, one, one, -4, 16),
        lambda: B.pages_assign(t, one, one, one, 4, 16, out=i32([[1], [2]])), lambda: B.pages_assign(i32([[0, 1], [2, 3]]).t(), one, one, one, 4, 16),
        lambda: B.pages_copy(k, None, t, k, k, t, one, 1), lambda: B.pages_copy(k, k, t, k[:1], k[:1], t, one, 1), lambda: B.pages_copy(k[0], k[1], t, k[0], k[1], t, one, 1),
        lambda: B.pages_copy(k, k, t, k, k, t, one, 2, row_idx=i32([[1]])), lambda: B.pages_copy(k, k, t, k, k, t, i32([1, 2]), 1),
        lambda: B.pages_copy(k, k, t, k, k, t, one, 2, row_idx=i32([1]), cu_idx=i32([0])),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(i))
    for status, call in ((-1, lambda: B.paged_attn(q, k[0], k[1], t, one, 0.1, max_kv_len=33)), (-1, lambda: B.paged_attn(q, k[0], k[1], t, one, 0.1, window=-1)),
                         (-3, lambda: B.paged_attn(q, k[0], k[1], t, one, 0.1, workspace=B.new_workspace(256))),
                         (-2, lambda: B.paged_attn(q, k[0].view(8, 8, 2, 64), k[1].view(8, 8, 2, 64), t, one, 0.1)),
                         (-1, lambda: B.rope_append(new, new, k[0], k[1], t, one, turns=B.rope_turns(128, 1e4))),
                         (-2, lambda: B.rope_append(new, new, k[0], k[1], t, one, turns=B.rope_turns(24, 1e4))),
                         (-2, lambda: B.pages_assign(t, one, one, one, 4, 20)), (-1, lambda: B.pages_copy(k, k, i32(np.zeros((0, 2))), k, k, t, one, 1))):
        with pytest.raises(B.SpecVLMError) as e:
            call()
        assert e.value.status == status


# ---------------------------------------------------------------------------------------------------- all of them together
def test_a_serving_loop(B):
    """Two requests decode with draft trees over paged caches: room for the block, positions and append, attention, greedy acceptance, the
    accepted rows to the front, the rest of the pages back, then a fork.  Beside it runs the same in plain NumPy over contiguous caches."""
    from paper_2508_16201_amd import synth
    hq, hkv, d, ps, n_pages, nodes, vocab, width = 8, 2, 64, 16, 40, 9, 64, 12
    rng = np.random.default_rng(0)
    bits = lambda *shape: synth.f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))
    turns, freq = B.rope_turns(d, 1e4), R.frequencies(d, 1e4)
    pool = [torch.full((1, n_pages, ps, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lens = [37, 20]
    table, *_, status = B.pages_assign(torch.full((2, width), -1, dtype=torch.int32, device="cuda"), i32([-1, -1]), i32([0, 0]), i32(lens), n_pages, ps)
    prompt = [bits(sum(lens), h, d) for h in (hkv, hkv)]
    B.rope_append(dev_bf16(prompt[0]), dev_bf16(prompt[1]), pool[0][0], pool[1][0], table, i32(lens), turns=turns, cu_q=i32([0, 37, 57]))
    tree = synth.make_tree(nodes, 5)
    depth = np.zeros(nodes, dtype=np.int64)
    for i in range(1, nodes):
        depth[i] = depth[tree[i]] + 1
    masks = np.asarray(synth.ancestor_masks(tree)).astype(np.uint64)

    def rows(b, n, held):                                                # what the pages hold of request b, as they are
        at = held.cpu().numpy()[b]
        j = np.arange(n)
        return [R.values(host_bits(p[0])[at[j // ps], j % ps]) for p in pool]

    context = [[x.copy() for x in rows(b, lens[b], table)] for b in range(2)]
    for step in range(4):
        grown = [n + nodes for n in lens]
        table, start, moved, refs, status = B.pages_assign(table, i32([0, 1]), i32(lens), i32(grown), n_pages, ps)
        assert status.tolist() == [0, 0] and moved.tolist() == [0, 0]
        q, k, v = bits(2 * nodes, hq, d), bits(2 * nodes, hkv, d), bits(2 * nodes, hkv, d)
        where = np.concatenate([n + depth for n in lens])
        turned = B.rope_append(dev_bf16(k), dev_bf16(v), pool[0][0], pool[1][0], table, i32(grown), q=dev_bf16(q), turns=turns, positions=i32(where))
        out = B.paged_attn(turned, pool[0][0], pool[1][0], table, i32(grown), 0.125, ancestor_mask=torch.from_numpy(np.tile(masks, 2).view(np.int64)).cuda())
        blocks = []
        for b in range(2):
            mine = slice(b * nodes, (b + 1) * nodes)
            kq, tol = R.rope(R.values(k[mine]), where[mine], freq, False, 1.0)
            have = rows(b, grown[b], table)
            assert np.array_equal(have[0][:lens[b]], context[b][0]) and np.array_equal(have[1][:lens[b]], context[b][1])
            assert (np.abs(have[0][lens[b]:] - kq) <= tol).all() and np.array_equal(have[1][lens[b]:], R.values(v[mine]))
            blocks.append([x[lens[b]:] for x in have])
            kb, vb = have[0], have[1]
            sees = [R.visible(grown[b], nodes, t, mask=masks[t]) for t in range(nodes)]
            for h in range(hq):
                want, _, off, _ = R.attention(host_f64(turned)[mine, h], kb[:, h // 4], vb[:, h // 4], 0.125, sees)
                assert (np.abs(host_f64(out)[mine, h] - want) <= off).all()
        # greedy acceptance of tokens that are often right
        target = rng.standard_normal((2, nodes, vocab)).astype(np.float32)
        tokens = rng.integers(0, vocab, (2, nodes)).astype(np.int32)
        for b in range(2):
            for i in range(1, nodes):
                if rng.random() < 0.7:
                    tokens[b, i] = target[b, tree[i]].argmax()
        n_acc, accepted, _ = B.accept_tree(torch.from_numpy(target).cuda(), torch.from_numpy(tokens).cuda(), torch.from_numpy(tree).cuda())
        base = i32(lens)
        B.pages_copy(*pool, table, *pool, table, n_acc, nodes, src_start=base, dst_start=base + 1, row_idx=accepted)
        lens_now = base + 1 + n_acc
        table, _, _, refs, status = B.pages_assign(table, i32([0, 1]), lens_now, lens_now, n_pages, ps)
        path = accepted.cpu().numpy()
        for b in range(2):
            n = int(n_acc[b])
            kept = [0] + [int(x) for x in path[b][:n]]
            context[b] = [np.concatenate([c, blk[kept]]) for c, blk in zip(context[b], blocks[b])]
            lens[b] += 1 + n
            assert lens[b] == int(lens_now[b])
            for have, want in zip(rows(b, lens[b], table), context[b]):
                assert np.array_equal(have, want)
        assert int(refs.sum()) == sum(-(-n // ps) for n in lens)
    # both go on from request 0, which is forked: each writes its own
    old = table
    n = lens[0]
    table, start, moved, refs, status = B.pages_assign(old, i32([0, 0]), i32([n, n]), i32([n + 1, n + 1]), n_pages, ps)
    B.pages_copy(*pool, old, *pool, table, moved, ps - 1, src_row=i32([0, 0]), src_start=start, dst_start=start)
    k, v = bits(2, hkv, d), bits(2, hkv, d)
    B.rope_append(dev_bf16(k), dev_bf16(v), pool[0][0], pool[1][0], table, i32([n + 1, n + 1]))
    for b in range(2):
        have = rows(b, n + 1, table)
        assert np.array_equal(have[0][:n], context[0][0]) and np.array_equal(have[1][:n], context[0][1])
        assert np.array_equal(have[0][n], R.values(k[b])) and np.array_equal(have[1][n], R.values(v[b]))
    assert refs.cpu().numpy().max() == 2


def test_a_window_that_moves_on(B):
    """A stream longer than its pages: what the window has passed is given up and used again."""
    hq, hkv, d, ps, n_pages, window, n_sinks, block, width = 4, 1, 64, 16, 6, 40, 4, 5, 40
    rng = np.random.default_rng(3)
    from paper_2508_16201_amd import synth
    bits = lambda *shape: synth.f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))
    pool = [torch.full((n_pages, ps, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    keys, values, n = np.zeros((0, hkv, d)), np.zeros((0, hkv, d)), 0
    for step in range(30):
        table, _, _, refs, status = B.pages_assign(table, i32([0]), i32([n]), i32([n + block]), n_pages, ps, window=window, n_sinks=n_sinks)
        assert status.item() == 0
        n += block
        q, k, v = bits(block, hq, d), bits(block, hkv, d), bits(block, hkv, d)
        B.rope_append(dev_bf16(k), dev_bf16(v), *pool, table, i32([n]))
        keys, values = np.concatenate([keys, R.values(k)]), np.concatenate([values, R.values(v)])
        out = B.paged_attn(dev_bf16(q), *pool, table, i32([n]), 0.125, window=window, n_sinks=n_sinks)
        sees = [R.visible(n, block, t, window, n_sinks) for t in range(block)]
        for h in range(hq):
            want, _, off, _ = R.attention(R.values(q)[:, h], keys[:, 0], values[:, 0], 0.125, sees)
            assert (np.abs(host_f64(out)[:, h] - want) <= off).all(), step
    assert n == 150 and int(refs.sum()) < n_pages


def test_assign_from_no_rows(B):
    """The first table of a program: nothing to go on from."""
    check_assign(B, np.zeros((0, 2), dtype=np.int32), [-1, -1], [0, 0], [20, 1], 5, 16)


def test_assign_for_no_rows(B):
    """The last request ended: every page is free, and the counts say so."""
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    junk = torch.full((1 << 20,), 7, dtype=torch.int32, device="cuda")
    del junk                                                                             # (what the next allocations find)
    table, start, rows, refs, status = B.pages_assign(i32([[0, 1]]), none, none, none, 700, 16)
    assert table.shape == (0, 2) and start.numel() == rows.numel() == status.numel() == 0
    assert refs.shape == (700,) and not refs.any()


def test_assign_refuses_a_table_over_the_old_one(B):
    both = torch.full((2, 6), -1, dtype=torch.int32, device="cuda")
    old, one = both[:, :3], i32([0, 1])
    for out in (old, both[:, 2:5], both[:, 1:4]):
        with pytest.raises(B.SpecVLMError) as e:
            B.pages_assign(old, one, i32([0, 0]), i32([5, 20]), 9, 16, out=out)
        assert e.value.status == -1
    B.pages_assign(old, one, i32([0, 0]), i32([5, 20]), 9, 16, out=both[:, 3:])          # side by side
    assert both.tolist() == [[-1, -1, -1, 0, -1, -1], [-1, -1, -1, 1, 2, -1]]


def test_copy_of_empty_lists(B):
    k = torch.ones((2, 4, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    t = i32([[0, 1], [2, 3]])
    B.pages_copy(v, v, t, k, k, t, None, 8, row_idx=torch.zeros(0, dtype=torch.int32, device="cuda"), cu_idx=i32([0, 0, 0]))
    assert (k == 1).all()


def test_turns_of_an_unknown_scaling(B):
    with pytest.raises(ValueError):
        B.rope_turns(64, 1e4, scaling="cubic")


@pytest.mark.parametrize("room", [8, 140])
def test_a_captured_step(B, room):
    """A whole step of two layers in one graph: room for the block, a fork's last page, positions and append, attention, rows to the front.  It is
    replayed over lengths and parents that change, each time beside the same calls made eagerly on a copy.  (room: pages a row, which
    decide the attention's variant)"""
    batch, layers, block, ps, n_pages = 3, 2, 4, 16, 64
    hq, hkv, d = 8, 2, 64
    torch.manual_seed(3)
    rnd = lambda *shape: torch.randn(shape, device="cuda").to(torch.bfloat16)
    q, k, v = rnd(layers, batch * block, hq, d), rnd(layers, batch * block, hkv, d), rnd(layers, batch * block, hkv, d)
    turns, idx = B.rope_turns(d, 1e4), i32([[0, 1, 3, 0], [0, 2, 0, 0], [0, 1, 2, 3]])
    counts, parent, keep, new = i32([3, 2, 4]), i32([0, 1, 2]), i32([0, 0, 0]), i32([block] * 3)
    pools = [rnd(layers, n_pages, ps, hkv, d) for _ in range(2)]
    table = torch.full((batch, room), -1, dtype=torch.int32, device="cuda")

    def step(pools, old, out):
        now, start, rows, refs, status = B.pages_assign(old, parent, keep, new, n_pages, ps, out=torch.empty_like(old))
        B.pages_copy(*pools, old, *pools, now, rows, ps - 1, src_row=parent, src_start=start, dst_start=start)
        for i in range(layers):
            turned = B.rope_append(k[i], v[i], pools[0][i], pools[1][i], now, new, q=q[i], turns=turns)
            B.paged_attn(turned, pools[0][i], pools[1][i], now, new, 0.125, out=out[i])
        first = new - block
        B.pages_copy(*pools, now, *pools, now, counts, block, src_start=first, dst_start=first, row_idx=idx)
        old.copy_(now)
        return refs, status

    out = torch.zeros_like(q)
    state = [x.clone() for x in pools], table.clone()
    step(*state, torch.zeros_like(out))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        refs, status = step(pools, table, out)
    state = [x.clone() for x in pools], table.clone()
    lens = [0, 0, 0]
    for parents, grow in (([-1, -1, -1], 40), ([0, 1, 2], 0), ([0, 0, 1], 7), ([2, 1, 1], 0), ([0, 1, 2], 23), ([1, 1, 1], 1)):
        kept = [lens[p] if p >= 0 else 0 for p in parents]
        lens = [n + block + grow for n in kept]
        for t, x in ((parent, parents), (keep, kept), (new, lens)):
            t.copy_(i32(x))
        graph.replay()
        want = torch.zeros_like(out)
        want_refs, want_status = step(*state, want)
        torch.cuda.synchronize()
        assert status.tolist() == [0, 0, 0] and torch.equal(refs, want_refs) and torch.equal(status, want_status)
        assert torch.equal(table, state[1])
        for a, b in zip([out] + pools, [want] + state[0]):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_two_calls_at_once(B):
    """Calls on two streams, each with what the binding allocates for it, over one cache that neither writes."""
    batch, n, ps, (hq, hkv, d) = 4, 3000, 16, (28, 4, 128)
    table, total = tables(1, [n] * batch, ps)
    torch.manual_seed(4)
    k, v = (torch.randn((total, ps, hkv, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    q = [torch.randn((batch * 3, hq, d), device="cuda").to(torch.bfloat16) for _ in range(2)]
    t, lens = i32(table), [i32([n, n - 7, 100, 3]), i32([2000, 5, n, n])]
    want = [B.paged_attn(a, k, v, t, b, 0.088) for a, b in zip(q, lens)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(B.paged_attn(q[i], k, v, t, lens[i], 0.088))
    torch.cuda.synchronize()
    for i in range(2):
        for x in got[i]:
            assert torch.equal(x.view(torch.int16), want[i].view(torch.int16))
