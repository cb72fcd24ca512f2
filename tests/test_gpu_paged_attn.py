"""specvlm_paged_attn against a plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

import paged_reference as R
from gpu_util import dev_bf16, host_f64, rnd_bits

pytestmark = pytest.mark.gpu
POISON = 0x7fc1                                     # a bf16 NaN: what rows that nobody wrote may hold
CROWD = 257                                         # more requests than CUs


@pytest.fixture(scope="module")
def B():
    from paper_2508_16201_amd import binding
    binding.lib()
    return binding


def build(seed, kv_lens, q_lens, heads, ps, spare=3, head_major=False, window=0, n_sinks=0, drop=(), pad_pages=0):
    """Requests' caches in pages in no order; rows and pages that belong to no token are poisoned.  drop: (request, page) that
    have been freed."""
    hq, hkv, d = heads
    rng = np.random.default_rng(seed)
    width = max(-(-n // ps) for n in kv_lens) + pad_pages
    held = [[i for i in range(-(-n // ps)) if (b, i) not in drop] for b, n in enumerate(kv_lens)]
    total = sum(len(h) for h in held) + spare
    ids, at = rng.permutation(total), 0
    table = np.full((len(kv_lens), width), -1, dtype=np.int32)
    k = np.full((total, ps, hkv, d), POISON, dtype=np.uint16)
    v = k.copy()
    for b, n in enumerate(kv_lens):
        for i in held[b]:
            page, rows = ids[at], min(ps, n - i * ps)
            at += 1
            table[b, i] = page
            k[page, :rows] = rnd_bits((rows, hkv, d), (seed, b, i, 1))
            v[page, :rows] = rnd_bits((rows, hkv, d), (seed, b, i, 2))
    q = rnd_bits((sum(q_lens), hq, d), (seed, 3))
    return q, k, v, table


def on_gpu(pool, head_major):
    if head_major:
        return dev_bf16(np.ascontiguousarray(pool.transpose(0, 2, 1, 3))).transpose(1, 2)
    return dev_bf16(pool)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def check(B, q, k, v, table, kv_lens, q_lens, scale, *, head_major=False, window=0, n_sinks=0, masks=None, ragged=None, max_kv_len=None, **kw):
    """The call against the plain implementation: as it is; among many requests with nothing to do, which leaves a workgroup to each; and unless
    the caller has a bound, with room for long caches, which takes launches that share a request's keys among workgroups."""
    ragged = len(set(q_lens)) > 1 if ragged is None else ragged
    more, crowd = dict(kw), dict(kw)
    cu_q = np.concatenate([[0], np.cumsum(q_lens)])
    crowd.update(cu_q=i32(np.concatenate([cu_q, [cu_q[-1]] * CROWD])), max_q_len=kw.get("max_q_len", max(q_lens)))
    if ragged:
        more.update(cu_q=i32(cu_q), max_q_len=crowd["max_q_len"])
    if masks is not None:
        more["ancestor_mask"] = crowd["ancestor_mask"] = torch.from_numpy(np.asarray(masks, dtype=np.uint64).view(np.int64)).cuda()
    qd = dev_bf16(q)
    want, want_lse, tol, tol_lse, written = R.paged_attention(R.values(q), R.values(k), R.values(v), table, kv_lens, q_lens, scale, window, n_sinks,
                                                              masks, max_kv_len)
    wide = np.concatenate([table, np.full((len(table), -(-8192 // k.shape[1])), -1, dtype=np.int32)], axis=1)
    many = np.concatenate([table, np.full((CROWD, table.shape[1]), -1, dtype=np.int32)])
    runs = [(many, list(kv_lens) + [0] * CROWD, crowd), (wide, kv_lens, more), (table, kv_lens, more)]
    for entries, lens, how in runs[:1] + runs[2:] if max_kv_len else runs:
        out = torch.full_like(qd, 7.0)
        got, lse = B.paged_attn(qd, on_gpu(k, head_major), on_gpu(v, head_major), i32(entries), i32(lens), scale, window=window, n_sinks=n_sinks,
                                out=out, want_lse=True, max_kv_len=max_kv_len, **how)
        torch.cuda.synchronize()
        assert got is out
        got, lse = host_f64(got), host_f64(lse)
        assert (got[~written] == 7.0).all()
        err = np.abs(got - want)[written]
        assert np.isfinite(got[written]).all()
        assert (err <= tol[written]).all(), (err - tol[written]).max()
        none = np.isinf(want_lse) & written[:, None]
        assert (lse[none] == -np.inf).all()
        some = ~none & written[:, None]
        assert (np.abs(lse[some] - want_lse[some]) <= tol_lse[some]).all()
    return got


HEADS = [(4, 1, 64), (14, 2, 64), (3, 3, 64), (28, 4, 128), (16, 2, 128), (5, 5, 128), (20, 1, 64)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("kv_len,q_len,ps", [(1, 1, 16), (2, 2, 16), (15, 1, 16), (16, 3, 16), (17, 5, 48), (63, 1, 16), (64, 4, 64), (65, 2, 64),
                                             (129, 7, 32), (200, 6, 96), (511, 1, 16), (777, 6, 256)])
def test_one_request(B, heads, kv_len, q_len, ps):
    q, k, v, table = build(kv_len * 31 + q_len, [kv_len], [q_len], heads, ps)
    check(B, q, k, v, table, [kv_len], [q_len], heads[2] ** -0.5)


@pytest.mark.parametrize("heads,kv_len,q_len", [((64, 8, 128), 3001, 6), ((14, 2, 64), 5003, 1), ((28, 4, 128), 2500, 1), ((8, 8, 64), 1511, 3)])
def test_split_and_joined(B, heads, kv_len, q_len):
    q, k, v, table = build(kv_len, [kv_len], [q_len], heads, 16)
    check(B, q, k, v, table, [kv_len], [q_len], heads[2] ** -0.5)


@pytest.mark.parametrize("heads,batch,kv_len", [((14, 2, 64), 1, n) for n in (512, 513, 1024, 1025, 1536, 1537)] + [((28, 4, 128), 1, n) for n in (512, 513, 832, 833)]
                         + [((16, 2, 128), 2, n) for n in (832, 833)] + [((8, 8, 64), 8, 40), ((8, 8, 64), 9, 40), ((3, 3, 64), 7, 200)])
def test_lengths_and_batches_between_the_kernels(B, heads, batch, kv_len):
    """The last size of one variant and the first of the next."""
    q, k, v, table = build(kv_len, [kv_len] * batch, [2] * batch, heads, 16)
    check(B, q, k, v, table, [kv_len] * batch, [2] * batch, heads[2] ** -0.5)


@pytest.mark.parametrize("window,n_sinks,q_len", [(1536 - 14 - 3 - 16, 16, 3), (1536 - 14 - 1, 0, 1), (1536 - 14 - 3, 1, 3), (512 - 14 - 2 - 32, 17, 2)])
def test_windows_that_fill_the_waves(B, window, n_sinks, q_len):
    """As many places as a window can have, at every offset of its first key in a group of 16."""
    kv_lens = [2600 + i for i in range(17)]
    for at in range(0, 17, 4):
        part = kv_lens[at:at + 4]
        q, k, v, table = build(window + at, part, [q_len] * len(part), (4, 1, 64), 16)
        check(B, q, k, v, table, part, [q_len] * len(part), 0.125, window=window, n_sinks=n_sinks)


@pytest.mark.parametrize("head_major", [False, True])
@pytest.mark.parametrize("heads", [(14, 2, 64), (8, 2, 128)])
def test_ragged_batch(B, heads, head_major):
    kv_lens, q_lens = [700, 1, 33, 64, 1290, 5], [6, 1, 4, 2, 1, 5]
    q, k, v, table = build(5, kv_lens, q_lens, heads, 32, pad_pages=2)
    check(B, q, k, v, table, kv_lens, q_lens, 0.1, head_major=head_major)


def test_more_requests_than_lanes(B):
    rng = np.random.default_rng(8)
    kv_lens = [int(n) for n in rng.integers(1, 200, 150)]
    q_lens = [min(n, int(m)) for n, m in zip(kv_lens, rng.integers(1, 4, 150))]
    q, k, v, table = build(8, kv_lens, q_lens, (4, 2, 64), 16)
    check(B, q, k, v, table, kv_lens, q_lens, 0.125)


def test_many_heads_and_requests_share_few_groups(B):
    kv_lens = [130, 260, 390, 64, 1]
    q, k, v, table = build(9, kv_lens, [1] * 5, (40, 40, 64), 16)
    check(B, q, k, v, table, kv_lens, [1] * 5, 0.125)


@pytest.mark.parametrize("tiles", [[4, 4, 4], [7, 5], [5, 5], [9, 9, 1], [6, 6, 6, 6, 6, 6], [1, 30, 1], [12, 0, 12], [2, 2, 2, 2, 2, 2, 2], [40, 41], [100, 96]])
@pytest.mark.parametrize("heads", [(40, 40, 64), (32, 32, 128)])
def test_requests_in_few_groups(B, heads, tiles):
    """Six or eight groups: runs from each request's first tile on, with a tile more, one request behind the other, several requests to a group."""
    kv_lens = [max(64 * n - 3 - i, 0) for i, n in enumerate(tiles)]
    q, k, v, table = build(sum(tiles), [max(n, 1) for n in kv_lens], [2] * len(tiles), heads, 16)
    check(B, q, k, v, table, kv_lens, [2] * len(tiles), heads[2] ** -0.5)


@pytest.mark.parametrize("q_len,heads", [(64, (4, 1, 64)), (33, (16, 2, 128)), (17, (4, 4, 128)), (12, (28, 4, 128)), (40, (3, 1, 128))])
def test_row_blocks_and_groups(B, q_len, heads):
    kv_lens = [300, 64 + q_len, q_len]
    q, k, v, table = build(q_len, kv_lens, [q_len] * 3, heads, 48)
    check(B, q, k, v, table, kv_lens, [q_len] * 3, heads[2] ** -0.5)


def test_padded_batch_leaves_the_rest_alone(B):
    """Requests with nothing to do, with lengths beyond the call's, and rows behind the last request."""
    kv_lens, q_lens = [50, 0, 20, 900, 3, 64], [2, 2, 0, 2, 5, 2]
    q, k, v, table = build(10, [max(n, 1) for n in kv_lens], q_lens + [3], (14, 2, 64), 16)
    check(B, q, k, v, table, kv_lens, q_lens, 0.125, max_kv_len=64, ragged=True)
    # without cu_q: an empty slot of a captured batch
    q, k, v, table = build(11, [50, 1, 20], [2] * 3, (14, 2, 64), 16)
    check(B, q, k, v, table, [50, 0, 20], [2] * 3, 0.125)


def trees(seed, q_lens):
    from paper_2508_16201_amd import synth
    return np.concatenate([np.asarray(synth.ancestor_masks(synth.make_tree(n, seed + i))).astype(np.uint64) for i, n in enumerate(q_lens)])


@pytest.mark.parametrize("heads", [(8, 2, 64), (16, 2, 128)])
def test_trees(B, heads):
    kv_lens, q_lens = [400, 26, 131], [26, 26, 9]
    q, k, v, table = build(12, kv_lens, q_lens, heads, 16)
    check(B, q, k, v, table, kv_lens, q_lens, heads[2] ** -0.5, masks=trees(1, q_lens))


def test_masks_that_leave_a_row_empty(B):
    """Query 0 of a block without context and a mask of nothing: 0, and -infinity in lse; a mask of 64 nodes."""
    q, k, v, table = build(13, [5, 64], [5, 64], (4, 2, 64), 16)
    masks = np.concatenate([[0, 1, 2, 0, 31], trees(2, [64])]).astype(np.uint64)
    masks[10] = 0
    got = check(B, q, k, v, table, [5, 64], [5, 64], 0.125, masks=masks)
    assert (got[[0, 3, 10]] == 0).all()


@pytest.mark.parametrize("window,n_sinks", [(1, 0), (1, 1), (16, 0), (17, 4), (100, 16), (100, 17), (64, 64), (250, 3), (5000, 4), (2 ** 31 - 1, 5), (33, 2 ** 31 - 1)])
def test_window_and_sinks(B, window, n_sinks):
    kv_lens, q_lens = [700, 3, 260, 64], [5, 3, 1, 8]
    q, k, v, table = build(window % 1000 + n_sinks % 1000, kv_lens, q_lens, (8, 2, 128), 16)
    check(B, q, k, v, table, kv_lens, q_lens, 0.088, window=window, n_sinks=n_sinks)


@pytest.mark.parametrize("heads", [(14, 2, 64), (8, 2, 128)])
@pytest.mark.parametrize("window,n_sinks", [(900, 0), (1500, 4), (2000, 130)])
def test_window_that_is_shared_among_workgroups(B, heads, window, n_sinks):
    kv_lens, q_lens = [2600], [5]
    q, k, v, table = build(window, kv_lens, q_lens, heads, 16)
    check(B, q, k, v, table, kv_lens, q_lens, heads[2] ** -0.5, window=window, n_sinks=n_sinks)


@pytest.mark.parametrize("ps", [16, 48, 256])
def test_window_over_freed_pages(B, ps):
    """What lies between the first keys and the window is in no page any more."""
    kv_lens, q_lens, window, n_sinks = [3001, 1500, 40], [4, 1, 2], 300, 5
    drop = {(b, i) for b, (n, m) in enumerate(zip(kv_lens, q_lens)) for i in range(-(-n // ps))
            if i * ps >= n_sinks and (i + 1) * ps <= n - m - window + 1}
    assert drop
    q, k, v, table = build(14, kv_lens, q_lens, (14, 2, 64), ps, drop=drop)
    check(B, q, k, v, table, kv_lens, q_lens, 0.125, window=window, n_sinks=n_sinks)


def test_window_in_a_tree(B):
    kv_lens, q_lens = [400, 100], [20, 12]
    q, k, v, table = build(15, kv_lens, q_lens, (8, 2, 64), 16)
    check(B, q, k, v, table, kv_lens, q_lens, 0.125, window=30, n_sinks=2, masks=trees(4, q_lens))


def test_pages_that_are_none_hide_their_keys(B):
    kv_lens, q_lens = [500, 70, 33], [3, 3, 1]
    q, k, v, table = build(16, kv_lens, q_lens, (8, 2, 128), 16, drop={(0, 0), (0, 7), (0, 8), (1, 2), (2, 0), (2, 1), (2, 2)})
    table[0, 7], table[1, 2] = len(k), 2 ** 31 - 1
    got = check(B, q, k, v, table, kv_lens, q_lens, 0.088)
    assert (got[6] == 0).all()                       # every key of the last request is hidden


def test_values_that_a_row_does_not_see_do_not_reach_it(B):
    """NaN and infinities in the keys and values of tree nodes and behind the window."""
    heads, kv_lens, q_lens = (8, 2, 128), [200, 90], [6, 6]
    q, k, v, table = build(17, kv_lens, q_lens, heads, 16)
    masks = np.array([1, 3, 5, 9, 17, 33] * 2, dtype=np.uint64)         # node i sees the root and itself
    wide = np.concatenate([table, np.full((2, 600), -1, dtype=np.int32)], axis=1)
    mask = torch.from_numpy(masks.view(np.int64)).cuda()
    many = np.concatenate([table, np.full((CROWD, table.shape[1]), -1, dtype=np.int32)])
    crowd = dict(cu_q=i32([0, 6] + [12] * (CROWD + 1)), max_q_len=6)
    for entries, lens, how in ((table, kv_lens, {}), (wide, kv_lens, {}), (many, kv_lens + [0] * CROWD, crowd)):
        run = lambda kk, vv, **more: host_f64(B.paged_attn(dev_bf16(q), dev_bf16(kk), dev_bf16(vv), i32(entries), i32(lens), 0.088, **how, **more))
        clean = run(k, v, ancestor_mask=mask)
        dirty = [x.copy() for x in (k, v)]
        for b, n in enumerate(kv_lens):
            for node, what in ((1, 0x7fc0), (3, 0x7f80), (5, 0xff80)):
                j = n - 6 + node
                for x in dirty:
                    x[table[b, j // 16], j % 16] = what
        got = run(*dirty, ancestor_mask=mask)
        for row in (0, 2, 4, 6, 8, 10):
            assert np.array_equal(got[row], clean[row]), row
        for row in (1, 3, 5, 7, 9, 11):
            assert not np.isfinite(got[row]).any(), row
        got = run(k, dirty[1], ancestor_mask=mask)                           # the values alone: what they are comes out
        assert np.isnan(got[[1, 7]]).all() and (got[[3, 9]] == np.inf).all() and (got[[5, 11]] == -np.inf).all()
        # behind the window, some of which the block's first query still sees
        window = 20
        base = run(k, v, window=window, n_sinks=3)
        dirty = [x.copy() for x in (k, v)]
        for b, n in enumerate(kv_lens):
            for j in [3, 15, 16] + list(range(n - 6 - window - 10, n - 6 - window + 1)) + [n - 6 - window + 2]:
                for x in dirty:
                    x[table[b, j // 16], j % 16] = 0x7f80
        got = run(*dirty, window=window, n_sinks=3)
        for b in range(2):
            assert not np.isfinite(got[6 * b]).any() and not np.isfinite(got[6 * b + 1]).any()
            assert np.array_equal(got[6 * b + 2:6 * b + 6], base[6 * b + 2:6 * b + 6])


def test_scale_zero_and_large(B):
    for scale in (0.0, 0.3):
        q, k, v, table = build(18, [90, 300], [2, 2], (8, 2, 64), 16)
        check(B, q, k, v, table, [90, 300], [2, 2], scale)


def test_logits_that_jump(B):
    """A key far above all before it, late in the cache, and a run of very low ones first."""
    q, k, v, table = build(19, [900], [2], (4, 1, 64), 16)
    kf = R.values(k)
    from paper_2508_16201_amd.synth import f32_to_bf16_bits
    for j in range(900):
        at = (table[0, j // 16], j % 16)
        f = 0.05 if j < 400 else 1.0
        kf[at] = kf[at] * f
    kf[table[0, 700 // 16], 700 % 16, 0] = 12 * R.values(q)[0, 0]
    k2 = f32_to_bf16_bits(np.nan_to_num(kf, nan=0.0).astype(np.float32))
    check(B, q, k2, v, table, [900], [2], 0.125)


def test_strides(B):
    """Pools and tables that are parts of larger tensors, queries with gaps between heads and tokens."""
    kv_lens, q_lens, heads = [200, 77], [3, 3], (8, 2, 64)
    q, k, v, table = build(20, kv_lens, q_lens, heads, 16)
    n = len(k)
    big = torch.zeros((2, n, 20, 5, 64), dtype=torch.bfloat16, device="cuda")
    kd, vd = big[0, :, 2:18, 1:5:2], big[1, :, 2:18, 1:5:2]
    kd.copy_(dev_bf16(k)); vd.copy_(dev_bf16(v))
    wide = torch.full((2, table.shape[1] + 9), 5, dtype=torch.int32, device="cuda")
    wide[:, 4:4 + table.shape[1]] = i32(table)
    qb = torch.zeros((6, 10, 128), dtype=torch.bfloat16, device="cuda")
    qd = qb[:, 1:9, 64:]
    qd.copy_(dev_bf16(q))
    out = torch.zeros_like(qb)[:, 1:9, 64:]
    B.paged_attn(qd, kd, vd, wide[:, 4:4 + table.shape[1]], i32(kv_lens), 0.125, out=out)           # (wide: rows of the table have a stride)
    plain = check(B, q, k, v, table, kv_lens, q_lens, 0.125)
    assert np.array_equal(host_f64(out), plain)


def test_pools_beyond_32_bits(B):
    """Pages whose bytes and elements lie past 2^32."""
    heads, ps = (8, 8, 128), 256
    kv_lens, q_lens = [600, 300], [2, 2]
    q, k, v, table = build(21, kv_lens, q_lens, heads, ps, spare=0)
    n = 2 ** 32 // (ps * 8 * 128) + 8
    kd = torch.empty((n, ps, 8, 128), dtype=torch.bfloat16, device="cuda")
    vd = torch.empty_like(kd)
    assert kd.numel() > 2 ** 32
    move = np.array([n - 1 - i for i in range(len(k))])
    kd[torch.from_numpy(move).cuda()] = dev_bf16(k)
    vd[torch.from_numpy(move).cuda()] = dev_bf16(v)
    got = B.paged_attn(dev_bf16(q), kd, vd, i32(np.where(table >= 0, move[table], -1)), i32(kv_lens), 0.088)
    assert np.array_equal(host_f64(got), check(B, q, k, v, table, kv_lens, q_lens, 0.088))


def test_same_as_over_a_contiguous_cache(B):
    """Within the roundings of both, what decode_attn and tree_attn say of the same keys."""
    hq, hkv, d, n, ql = 28, 4, 128, 2777, 6
    q, k, v, table = build(22, [n], [ql], (hq, hkv, d), 16, spare=0)
    rows = np.arange(n)
    kc, vc = (dev_bf16(x[table[0, rows // 16], rows % 16]) for x in (k, v))
    mask = torch.from_numpy(trees(3, [ql]).view(np.int64)).cuda()
    for more in ({}, {"ancestor_mask": mask}):
        a = host_f64(B.decode_attn(dev_bf16(q), kc, vc, 0.088, **more))
        b = host_f64(B.paged_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), i32(table), i32([n]), 0.088, **more))
        _, _, tol, _, _ = R.paged_attention(R.values(q), R.values(k), R.values(v), table, [n], [ql], 0.088,
                                            masks=trees(3, [ql]) if more else None)
        # (decode_attn rounds its probabilities and its partial results to bf16 on the way: 2^-8 each of the terms, whose sum of
        # sizes is at most the largest value)
        assert (np.abs(a - b) <= 2 * tol + 2 * 2.0 ** -8 * np.nanmax(np.abs(R.values(v)))).all()


@pytest.mark.parametrize("room", [1500, 8000])
def test_runs_are_alike_and_replays_follow_the_lengths(B, room):
    """A captured call over caches that grow, with eager calls between the replays; the workspace is poisoned."""
    heads, ps, q_len = (14, 2, 64), 16, 3
    kv_lens = [400, 35, 1500]
    q, k, v, table = build(23, kv_lens, [q_len] * 3, heads, ps)
    wide = np.concatenate([table, np.full((3, 8000 // ps - table.shape[1]), -1, dtype=np.int32)], axis=1)
    qd, kd, vd, td = dev_bf16(q), dev_bf16(k), dev_bf16(v), i32(wide)
    lens = i32([3, 3, 3])
    ws = B.new_workspace(B.paged_attn_workspace_bytes(3, q_len, *heads))
    out = torch.empty_like(qd)
    call = lambda o, w: B.paged_attn(qd, kd, vd, td, lens, 0.125, max_kv_len=room, out=o, workspace=w)
    call(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    for now in ([3, 3, 3], [100, 4, 900], [400, 35, 1500], [400, 0, 7], [64, 35, 1473]):
        lens.copy_(i32(now))
        ws.fill_(255)
        out.fill_(0)
        graph.replay()
        eager = torch.zeros_like(qd)
        call(eager, None)
        again = torch.zeros_like(qd)
        call(again, None)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16)), now
        assert torch.equal(again.view(torch.int16), eager.view(torch.int16)), now
        want, _, tol, _, written = R.paged_attention(R.values(q), R.values(k), R.values(v), table, now, [q_len] * 3, 0.125)
        assert (np.abs(host_f64(out) - want)[written] <= tol[written]).all()
        assert (host_f64(out)[~written] == 0).all()


def test_on_another_stream(B):
    q, k, v, table = build(24, [900], [4], (16, 2, 128), 32)
    want = check(B, q, k, v, table, [900], [4], 0.088)
    side = torch.cuda.Stream()
    kd, vd, td, ld = dev_bf16(k), dev_bf16(v), i32(table), i32([900])
    base = dev_bf16(q)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        qd = base * 1
        got = B.paged_attn(qd, kd, vd, td, ld, 0.088)
    side.synchronize()
    assert np.array_equal(host_f64(got), want)


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(B, seed):
    rng = np.random.default_rng(1000 + seed)
    heads = HEADS[rng.integers(len(HEADS))]
    batch, ps = int(rng.integers(1, 7)), int(rng.choice([16, 32, 48, 64, 128]))
    top = int(rng.choice([1, 3, 8, 30]))
    kv_lens = [int(np.exp(rng.uniform(0, np.log(900)))) for _ in range(batch)]
    q_lens = [min(n, int(rng.integers(1, top + 1))) for n in kv_lens]
    q, k, v, table = build(2000 + seed, kv_lens, q_lens, heads, ps)
    window = int(rng.integers(1, 400)) if rng.random() < 0.4 else 0
    masks = trees(seed, q_lens) if rng.random() < 0.3 else None
    check(B, q, k, v, table, kv_lens, q_lens, heads[2] ** -0.5, window=window, n_sinks=int(rng.integers(0, 40)), masks=masks,
          head_major=bool(rng.random() < 0.5))
