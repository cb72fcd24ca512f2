"""The operators for many texts over one video as the host sees them: refusals before any launch, workspace sizes, what a call launches, and the plain
implementations that the kernels are held to.  No GPU is touched."""
import os

import numpy as np
import pytest

import launches as L
import paged_reference as R
import shared_reference as S

AT = L.AT


@pytest.fixture(scope="module")
def B():
    from paper_2508_16201_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding


SHARED = dict(page_table=AT, table_stride=50, max_pages=50, n_pages=100, page_size=16, kv_lens=AT, batch=3, q_len=2, min_tokens=16, groups=AT, workspace=AT,
              workspace_bytes=1 << 40)
ATTN = dict(q=AT, q_tok_stride=1792, q_head_stride=128, k_pages=AT, v_pages=AT, page_stride=16 * 512, tok_stride=512, head_stride=128, n_pages=100,
            page_size=16, page_table=AT, table_stride=50, max_pages=50, kv_lens=AT, groups=AT, batch=3, n_queries=6, q_len=2, kv_len=800, n_q_heads=28,
            n_kv_heads=4, head_dim=128, softmax_scale=0.1, out=AT, workspace=AT, workspace_bytes=1 << 40)
CROSS = dict(q=AT, q_tok_stride=1792, q_head_stride=128, k=AT, v=AT, kv_tok_stride=512, kv_head_stride=128, cu_q=AT, cu_kv=AT, batch=3, n_queries=6,
             n_states=800, n_q_heads=28, n_kv_heads=4, head_dim=128, softmax_scale=0.1, out=AT, workspace=AT, workspace_bytes=1 << 40)
CALLS = {"specvlm_pages_shared": SHARED, "specvlm_shared_attn": ATTN, "specvlm_cross_attn": CROSS}

REFUSED = [
    # (function, what is changed, status)
    *[("specvlm_pages_shared", {k: None}, -1) for k in ("page_table", "kv_lens", "groups")],
    *[("specvlm_pages_shared", {k: -1}, -1) for k in ("batch", "q_len", "n_pages", "max_pages", "min_tokens", "table_stride")],
    ("specvlm_pages_shared", {"page_size": 0}, -1), ("specvlm_pages_shared", {"page_size": 40}, -2), ("specvlm_pages_shared", {"batch": 8193}, -2),
    ("specvlm_pages_shared", {"batch": 8192}, 0), ("specvlm_pages_shared", {"max_pages": 1 << 27, "page_size": 16}, -2),
    ("specvlm_pages_shared", {"max_pages": (1 << 27) - 1, "page_size": 16}, 0), ("specvlm_pages_shared", {"workspace": None}, -3),
    ("specvlm_pages_shared", {"workspace": AT + 4}, -3), ("specvlm_pages_shared", {"workspace_bytes": 11}, -3),
    *[("specvlm_shared_attn", {k: None}, -1) for k in ("q", "k_pages", "v_pages", "page_table", "kv_lens", "groups", "out")],
    *[("specvlm_shared_attn", {k: -1}, -1) for k in ("batch", "n_queries", "q_len", "kv_len", "n_pages", "max_pages", "table_stride")],
    ("specvlm_shared_attn", {"n_q_heads": 27}, -1), ("specvlm_shared_attn", {"n_kv_heads": 0}, -1), ("specvlm_shared_attn", {"page_size": 0}, -1),
    ("specvlm_shared_attn", {"softmax_scale": -1.0}, -1), ("specvlm_shared_attn", {"softmax_scale": float("nan")}, -1),
    ("specvlm_shared_attn", {"softmax_scale": float("inf")}, -1), ("specvlm_shared_attn", {"n_queries": 7}, -1), ("specvlm_shared_attn", {"n_queries": 7, "cu_q": AT}, 0),
    ("specvlm_shared_attn", {"kv_len": 801}, -1), ("specvlm_shared_attn", {"kv_len": 1}, -1), ("specvlm_shared_attn", {"n_pages": 0}, -1),
    ("specvlm_shared_attn", {"head_dim": 96}, -2), ("specvlm_shared_attn", {"page_size": 24}, -2),
    ("specvlm_shared_attn", {"q_len": 65, "n_queries": 195, "ancestor_mask": AT}, -2), ("specvlm_shared_attn", {"q_len": 65, "n_queries": 195}, 0),
    ("specvlm_shared_attn", {"q_len": 64, "n_queries": 192, "ancestor_mask": AT}, 0),
    *[("specvlm_shared_attn", {k: 12}, -2) for k in ("q_tok_stride", "q_head_stride", "page_stride", "tok_stride", "head_stride")],
    *[("specvlm_shared_attn", {k: AT + 8}, -2) for k in ("q", "k_pages", "v_pages", "out")],
    ("specvlm_shared_attn", {"tok_stride": 1 << 26}, -2), ("specvlm_shared_attn", {"tok_stride": -8}, -2),
    ("specvlm_shared_attn", {"page_size": 1 << 26, "kv_len": (1 << 30) + 1}, -2), ("specvlm_shared_attn", {"workspace": None}, -3),
    ("specvlm_shared_attn", {"workspace": AT + 16}, -3), ("specvlm_shared_attn", {"workspace_bytes": 1000}, -3),
    # rows, rows of partial results and work are 32-bit numbers
    ("specvlm_shared_attn", {"cu_q": AT, "n_queries": (1 << 29) // 28 + 1}, -2), ("specvlm_shared_attn", {"cu_q": AT, "batch": 1 << 22}, -2),
    ("specvlm_shared_attn", {"cu_q": AT, "batch": 1 << 20, "page_size": 1 << 20, "kv_len": 1 << 24}, -2),
    *[("specvlm_cross_attn", {k: None}, -1) for k in ("q", "k", "v", "out", "cu_q", "cu_kv")],
    *[("specvlm_cross_attn", {k: -1}, -1) for k in ("batch", "n_queries", "n_states", "n_q_heads", "n_kv_heads")],
    ("specvlm_cross_attn", {"cu_q": None, "cu_kv": None}, -1), ("specvlm_cross_attn", {"cu_q": None, "cu_kv": None, "batch": 1}, 0),
    ("specvlm_cross_attn", {"n_q_heads": 27}, -1), ("specvlm_cross_attn", {"softmax_scale": -1.0}, -1), ("specvlm_cross_attn", {"softmax_scale": float("nan")}, -1),
    ("specvlm_cross_attn", {"head_dim": 80}, -2), ("specvlm_cross_attn", {"n_states": 0}, 0), ("specvlm_cross_attn", {"n_states": 0, "k": None, "v": None}, 0),
    ("specvlm_cross_attn", {"n_states": (1 << 30) + 1}, -2),
    *[("specvlm_cross_attn", {k: 12}, -2) for k in ("q_tok_stride", "q_head_stride", "kv_tok_stride", "kv_head_stride")],
    *[("specvlm_cross_attn", {k: AT + 8}, -2) for k in ("q", "k", "v", "out")],
    ("specvlm_cross_attn", {"kv_tok_stride": 1 << 26}, -2), ("specvlm_cross_attn", {"workspace": None}, -3), ("specvlm_cross_attn", {"workspace": AT + 16}, -3),
    ("specvlm_cross_attn", {"workspace_bytes": 1000}, -3), ("specvlm_cross_attn", {"n_queries": (1 << 29) // 28 + 1}, -2),
    ("specvlm_cross_attn", {"n_queries": 1 << 20, "n_states": 1 << 27}, -2),
]
NOTHING = [("specvlm_pages_shared", {"batch": 0, "workspace": None}), ("specvlm_shared_attn", {"batch": 0}), ("specvlm_shared_attn", {"q_len": 0, "n_queries": 0}),
           ("specvlm_shared_attn", {"cu_q": AT, "n_queries": 0}), ("specvlm_cross_attn", {"batch": 0}), ("specvlm_cross_attn", {"n_queries": 0})]


def test_refusals_launch_nothing(tmp_path):
    got = L.launches([(f, {**CALLS[f], **change}) for f, change, _ in REFUSED] + [(f, {**CALLS[f], **change}) for f, change in NOTHING], tmp_path)
    for (f, change, want), (status, launched) in zip(REFUSED, got):
        assert status == want, (f, change, status)
        assert want == 0 or not launched, (f, change)
    for (f, change), (status, launched) in zip(NOTHING, got[len(REFUSED):]):
        assert status == 0 and not launched, (f, change, status, launched)


def test_launches(tmp_path):
    """No launch has 2^32 threads, and none asks for more LDS than a CU has."""
    big = {**ATTN, "cu_q": AT, "n_queries": (1 << 26) // 28, "batch": 2, "kv_len": 16, "q_len": 16}
    got = L.launches([("specvlm_pages_shared", SHARED), ("specvlm_pages_shared", {**SHARED, "batch": 8192}), ("specvlm_shared_attn", ATTN), ("specvlm_cross_attn", CROSS), ("specvlm_shared_attn", big),
                      ("specvlm_shared_attn", {**ATTN, "head_dim": 64})], tmp_path)
    for status, launched in got:
        assert status == 0 and launched
        for kernel, grid, block, lds, *_ in launched:
            assert np.prod(grid, dtype=np.int64) * np.prod(block, dtype=np.int64) < 2 ** 32 and lds <= 160 * 1024, (kernel, grid, block, lds)


def test_a_launch_that_fails_is_said(tmp_path):
    got = L.launches([(f, {**args, "batch": 20} if f == "specvlm_pages_shared" else args, 1) for f, args in CALLS.items()], tmp_path)
    assert [status for status, _ in got] == [-4] * 3


def test_workspace_queries(B):
    assert B.pages_shared_workspace_bytes(3) > 0 and B.pages_shared_workspace_bytes(0) == 0 and B.pages_shared_workspace_bytes(8193) == 0
    for f in (B.shared_attn_workspace_bytes, B.cross_attn_workspace_bytes):
        assert f(3, 6, 28, 4, 128) > 0
        for bad in ((3, 6, 28, 4, 96), (0, 6, 28, 4, 128), (3, 0, 28, 4, 128), (3, 6, 27, 4, 128), (-1, 6, 28, 4, 128), (3, 6, 0, 4, 128), (3, 6, 28, 0, 128)):
            assert f(*bad) == 0


def test_the_binding_refuses_what_does_not_fit(B):
    import torch
    k, v = (torch.zeros(4, 16, 2, 64).bfloat16() for _ in range(2))
    i, g = torch.zeros(1, dtype=torch.int32), torch.zeros((3, 1), dtype=torch.int32)
    for call in (lambda: B.shared_attn(torch.zeros(1, 4, 64).bfloat16(), k, v, i[None], i, 0.1, g),
                 lambda: B.pages_shared(i[None], i, 4, 16, 1), lambda: B.cross_attn(torch.zeros(1, 4, 64).bfloat16(), k[0], v[0], 0.1)):
        with pytest.raises(ValueError):
            call()


def test_plain_attention_is_the_paged_ones(oracle_lib):
    """Blocks over pages, chain and tree, as the plain implementation of paged attention has them; cross attention of one block's context as the oracle has it."""
    rng = np.random.default_rng(1)
    from paper_2508_16201_amd import synth
    q, k, v = (synth.f32_to_bf16_bits(rng.standard_normal(s).astype(np.float32)) for s in ((5, 4, 64), (48, 2, 64), (48, 2, 64)))
    table = np.array([[2, 0, 1]], dtype=np.int32)
    pages = [R.values(x).reshape(3, 16, 2, 64) for x in (k, v)]
    masks = np.asarray(synth.ancestor_masks(synth.make_tree(5, 3))).astype(np.uint64)
    for m in (None, masks):
        out, lse, _, _, _ = S.shared_attention(R.values(q), *pages, table, [40], [5], 0.125, masks=m)
        want, want_lse, _, _, _ = R.paged_attention(R.values(q), *pages, table, [40], [5], 0.125, masks=m)
        assert np.allclose(out, want, atol=1e-12) and np.allclose(lse, want_lse, atol=1e-12)
    # a block's last query sees all of its keys
    want, want_lse = oracle_lib.decode_attn(q[4:], k, v, 0.125)
    out, lse, _, _ = S.cross_attention(R.values(q[4:]), R.values(k), R.values(v), [1], [48], 0.125)
    assert np.allclose(out, want, atol=1e-12) and np.allclose(lse, want_lse, atol=1e-12)
    out, lse, _, _ = S.cross_attention(R.values(q), R.values(k), R.values(v), [2, 3], [0, 48], 0.125, np.array([[0, 9]] * 4 + [[7, 7]]))
    assert (out[[0, 1, 4]] == 0).all() and (lse[[0, 1, 4]] == -np.inf).all() and np.isfinite(lse[2:4]).all()


def test_plain_groups():
    """By hand: c = 0 3 3 1 2 0 (pages of 16)."""
    table = np.array([[1, 2, 3, 4], [1, 2, 3, 5], [1, 2, 3, 6], [1, 7, 8, 9], [1, 7, 9, 9], [4, 4, 4, 4]])
    lens, blocks = [64] * 6, [3] * 6
    assert S.groups(table, lens, blocks, 10, 16, 0).tolist() == [[0, 0, 0, 3, 3, 5], [3, 0, 0, 2, 0, 1], [48, 48, 48, 32, 32, 0]]
    assert S.groups(table, lens, blocks, 10, 16, 33).tolist() == [[0, 0, 0, 3, 4, 5], [3, 0, 0, 1, 1, 1], [48, 48, 48, 0, 0, 0]]
    assert S.groups(table, [64, 34, 64, 64, 64, 64], blocks, 10, 16, 0).tolist() == [[0, 0, 0, 0, 0, 5], [5, 0, 0, 0, 0, 1], [16] * 5 + [0]]
    # (two pages of the first rows are pages of a pool of three, then one: c = 0 2 2 1 1 0)
    assert S.groups(table, lens, blocks, 3, 16, 0).tolist() == [[0, 0, 0, 0, 0, 5], [5, 0, 0, 0, 0, 1], [16] * 5 + [0]]
