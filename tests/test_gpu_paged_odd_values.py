"""specvlm_paged_attn over values that are no finite numbers (what a row sees of them comes out, wherever their keys lie, and what it does
not see changes no bit of it), and over values too large for a product with an early maximum's probability."""
import numpy as np
import pytest
import torch

import paged_reference as R
from gpu_util import dev_bf16, host_f64
from test_gpu_paged_attn import CROWD, build, i32, on_gpu

pytestmark = pytest.mark.gpu
INF, DOWN, NAN = 0x7f80, 0xff80, 0x7fc0


@pytest.fixture(scope="module")
def B():
    from paper_2508_16201_amd import binding
    binding.lib()
    return binding


def bits(x):
    from paper_2508_16201_amd.synth import f32_to_bf16_bits
    return f32_to_bf16_bits(np.asarray(x, dtype=np.float32))


def at(table, b, ps, j):
    return table[b, j // ps], j % ps


def variants(table, kv_lens, q_lens, ps):
    """The call as it is; with room for long caches (keys shared among workgroups); among many requests (a workgroup has one whole)."""
    wide = np.concatenate([table, np.full((len(table), -(-8192 // ps)), -1, dtype=np.int32)], axis=1)
    many = np.concatenate([table, np.full((CROWD, table.shape[1]), -1, dtype=np.int32)])
    cu_q = np.concatenate([[0], np.cumsum(q_lens)])
    crowd = dict(cu_q=i32(np.concatenate([cu_q, [cu_q[-1]] * CROWD])), max_q_len=max(q_lens))
    return {"short": (table, kv_lens, {}), "shared": (wide, kv_lens, {}), "whole": (many, list(kv_lens) + [0] * CROWD, crowd)}


def check(B, q, k, v, table, kv_lens, q_lens, scale, odd, *, what=None, **more):
    """odd: what columns hold (inf, -inf or nan), in every head; the others are held to 64 bits over values that are 0 in the odd places."""
    ps = k.shape[1]
    flat = v.copy()
    flat[~np.isfinite(R.values(v))] = 0
    want, want_lse, tol, tol_lse, _ = R.paged_attention(R.values(q), R.values(k), R.values(flat), table, kv_lens, q_lens, scale, **more)
    plain = [c for c in range(q.shape[2]) if c not in odd]
    for name, (entries, lens, how) in variants(table, kv_lens, q_lens, ps).items():
        if what and name not in what:
            continue
        got, lse = B.paged_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), i32(entries), i32(lens), scale, want_lse=True, **how, **more)
        got, lse = host_f64(got), host_f64(lse)
        assert (np.abs(got - want)[:, :, plain] <= tol[:, :, plain]).all(), name
        assert (np.abs(lse - want_lse) <= tol_lse).all(), name
        for c, x in odd.items():
            assert np.isnan(got[:, :, c]).all() if np.isnan(x) else (got[:, :, c] == x).all(), (name, c, x, got[:, :, c])


@pytest.mark.parametrize("heads,q_len", [((8, 2, 128), 1), ((8, 2, 128), 6), ((64, 8, 128), 6), ((16, 1, 128), 4), ((4, 1, 64), 1), ((14, 2, 64), 3),
                                         ((16, 2, 64), 6), ((16, 1, 64), 4)])
def test_values_that_every_row_sees(B, heads, q_len):
    """Far before the block, where no mask is near."""
    kv_lens, q_lens = [500, 300], [q_len] * 2
    q, k, v, table = build(31 + q_len, kv_lens, q_lens, heads, 16)
    for b in range(2):
        for j, c, x in ((37, 0, INF), (37, 1, DOWN), (101, 2, NAN), (40, 3, INF), (170, 3, DOWN), (33, 4, INF), (250, 4, INF), (5, 63, DOWN)):
            v[at(table, b, 16, j)][:, c] = x
    check(B, q, k, v, table, kv_lens, q_lens, heads[2] ** -0.5, {0: np.inf, 1: -np.inf, 2: np.nan, 3: np.nan, 4: np.inf, 63: -np.inf})


def test_values_inside_a_window(B):
    heads, kv_lens, q_lens = (8, 2, 128), [500, 300], [3, 3]
    q, k, v, table = build(32, kv_lens, q_lens, heads, 16)
    for b, n in enumerate(kv_lens):
        for j, c, x in ((n - 100, 0, INF), (n - 131, 1, DOWN), (2, 2, INF), (n - 201, 3, INF), (6, 5, DOWN)):
            v[at(table, b, 16, j)][:, c] = x                                 # (the last two: between the first keys and every window)
    check(B, q, k, v, table, kv_lens, q_lens, 0.088, {0: np.inf, 1: -np.inf, 2: np.inf}, window=180, n_sinks=4)


@pytest.mark.parametrize("heads,ps", [((16, 2, 64), 48), ((16, 2, 128), 32)])
def test_values_in_pools_by_heads_with_pages_that_are_none(B, heads, ps):
    """Keys of a missing page are hidden in the second look too, whatever lies in the pool's first page."""
    kv_lens, q_lens = [600, 300], [3, 3]
    q, k, v, table = build(36, kv_lens, q_lens, heads, ps, drop={(0, 1), (0, 5), (1, 2)})
    for b in range(2):
        for j, c, x in ((7, 0, INF), (7, 1, DOWN), (ps * 4 + 3, 2, NAN)):
            v[at(table, b, ps, j)][:, c] = x
    flat = v.copy()
    flat[~np.isfinite(R.values(v))] = 0
    want, _, tol, _, _ = R.paged_attention(R.values(q), R.values(k), R.values(flat), table, kv_lens, q_lens, 0.1)
    kd, vd = on_gpu(k, True), on_gpu(v, True)
    for name, (entries, lens, how) in variants(table, kv_lens, q_lens, ps).items():
        got = host_f64(B.paged_attn(dev_bf16(q), kd, vd, i32(entries), i32(lens), 0.1, **how))
        assert (got[:, :, 0] == np.inf).all() and (got[:, :, 1] == -np.inf).all() and np.isnan(got[:, :, 2]).all(), name
        assert (np.abs(got - want)[:, :, 3:] <= tol[:, :, 3:]).all(), name


@pytest.mark.parametrize("heads", [(3, 3, 64), (5, 5, 128)])
@pytest.mark.parametrize("low,odd_at", [((0, 350), 20), ((350, 690), 600), ((0, 690), 300)])
def test_values_of_small_weight(B, heads, low, odd_at):
    """Keys with logits of -400, whose weight 32 bits take for 0, hold the infinities: before the others, behind them, in other pieces."""
    hq, hkv, d = heads
    scale, n = d ** -0.5, 700
    q, k, v, table = build(33, [n], [1], heads, 16)
    qf = R.values(q)[0]
    far = bits(-400 * qf / (qf ** 2).sum(1, keepdims=True) / scale)
    for j in range(*low):
        k[at(table, 0, 16, j)] = far
    v[at(table, 0, 16, odd_at)][:, 0] = INF
    v[at(table, 0, 16, odd_at)][:, 1] = DOWN
    v[at(table, 0, 16, odd_at + 1)][:, 2] = NAN
    check(B, q, k, v, table, [n], [1], scale, {0: np.inf, 1: -np.inf, 2: np.nan})


@pytest.mark.parametrize("heads", [(16, 2, 128), (16, 1, 64)])
def test_values_that_one_row_sees_do_not_touch_the_others(B, heads):
    """A tree's node with an infinite value, and one before every mask that all rows see: columns and rows without it stay bit for bit."""
    kv_lens, q_lens = [500, 300], [4, 4]
    q, k, v, table = build(35, kv_lens, q_lens, heads, 16)
    mask = torch.tensor([1, 3, 5, 9] * 2, dtype=torch.int64).cuda()
    for name, (entries, lens, how) in variants(table, kv_lens, q_lens, 16).items():
        run = lambda vv: host_f64(B.paged_attn(dev_bf16(q), dev_bf16(k), dev_bf16(vv), i32(entries), i32(lens), 0.088, ancestor_mask=mask, **how))
        clean, dirty = run(v), v.copy()
        for b, n in enumerate(kv_lens):
            dirty[at(table, b, 16, n - 3)][:, 0] = INF                     # node 1: row 1 alone
            dirty[at(table, b, 16, 64)][:, 5] = DOWN
        got = run(dirty)
        assert (got[[1, 5], :, 0] == np.inf).all() and (got[:, :, 5] == -np.inf).all(), name
        got[[1, 5], :, 0], clean[[1, 5], :, 0] = 0, 0
        got[:, :, 5], clean[:, :, 5] = 0, 0
        assert np.array_equal(got, clean), name


@pytest.mark.parametrize("heads,n,what", [((3, 3, 64), 700, ("short", "whole")), ((5, 5, 128), 440, ("short", "whole")), ((5, 5, 128), 9000, ("short",)),
                                          ((4, 4, 64), 20000, ("short",))])
def test_large_values_behind_a_small_maximum(B, heads, n, what):
    """A key whose logit is 62 over those before it, with values of 2^60: its probability against the early maximum, 2^89, times that is too
    large for 32 bits, the sum divided by its normaliser is not."""
    hq, hkv, d = heads
    scale = d ** -0.5
    q, k, v, table = build(34, [n], [1], heads, 16)
    qf = R.values(q)[0]
    high = bits(62 * qf / (qf ** 2).sum(1, keepdims=True) / scale)
    for j in range(150, n - 20, 800):
        k[at(table, 0, 16, j)] = high
        v[at(table, 0, 16, j)][:, :3] = bits([2.0 ** 60, -2.0 ** 61, 1.5 * 2.0 ** 60])
    check(B, q, k, v, table, [n], [1], scale, {}, what=what)
