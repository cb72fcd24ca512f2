"""specvlm_paged_attn where its operands lie: an output over the queries."""
import numpy as np
import pytest

import paged_reference as R
from gpu_util import dev_bf16, host_f64
from test_gpu_paged_attn import build, i32
from test_gpu_paged_odd_values import variants

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2508_16201_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("heads,q_len", [((14, 2, 64), 1), ((8, 2, 128), 6), ((64, 8, 128), 6), ((16, 1, 64), 20)])
def test_an_output_over_the_queries(B, heads, q_len):
    kv_lens, q_lens = [500, 300], [q_len] * 2
    q, k, v, table = build(41 + q_len, kv_lens, q_lens, heads, 16)
    kd, vd = dev_bf16(k), dev_bf16(v)
    want, _, tol, _, _ = R.paged_attention(R.values(q), R.values(k), R.values(v), table, kv_lens, q_lens, 0.1)
    for name, (entries, lens, how) in variants(table, kv_lens, q_lens, 16).items():
        qd = dev_bf16(q)
        over = B.paged_attn(qd, kd, vd, i32(entries), i32(lens), 0.1, out=qd, **how)
        assert over is qd
        assert (np.abs(host_f64(over) - want) <= tol).all(), name
        if name != "short":                                    # (which is another kernel then)
            assert np.array_equal(host_f64(over), host_f64(B.paged_attn(dev_bf16(q), kd, vd, i32(entries), i32(lens), 0.1, **how))), name


@pytest.mark.parametrize("heads,window", [((14, 2, 64), 0), ((8, 2, 128), 0), ((8, 2, 128), 40)])
def test_entries_behind_the_last_token(B, heads, window):
    """Ids of pages that hold NaN, of other requests' pages and of none: results are those of a table that ends."""
    kv_lens, q_lens = [500, 33, 257], [3, 3, 1]
    q, k, v, table = build(43, kv_lens, q_lens, heads, 16, spare=5, pad_pages=7)
    free = np.setdiff1d(np.arange(len(k)), table)                  # pages of nobody: NaN throughout
    stale = table.copy()
    for b, n in enumerate(kv_lens):
        behind = -(-n // 16)
        stale[b, behind:] = np.resize([*free, table[0, 0], len(k), 2 ** 31 - 1, -7, table[2, 1]], table.shape[1] - behind)
    kd, vd, qd = dev_bf16(k), dev_bf16(v), dev_bf16(q)
    cu_q = i32([0, 3, 6, 7])
    for (name, (clean, lens, how)), (_, (dirty, _, _)) in zip(variants(table, kv_lens, q_lens, 16).items(), variants(stale, kv_lens, q_lens, 16).items()):
        how = how or dict(cu_q=cu_q, max_q_len=3)
        run = lambda entries: B.paged_attn(qd, kd, vd, i32(entries), i32(lens), 0.1, window=window, n_sinks=3, want_lse=True, **how)
        (a, a_lse), (b, b_lse) = run(clean), run(dirty)
        assert np.array_equal(host_f64(a), host_f64(b)) and np.array_equal(host_f64(a_lse), host_f64(b_lse)), name
        assert np.isfinite(host_f64(a)).all(), name
