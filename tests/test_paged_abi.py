"""The paged operators as the host sees them: refusals before any launch, workspace sizes, what a call launches, and the
frequencies of rotary positions.  No GPU is touched."""
import ctypes as C
import os

import numpy as np
import pytest

import launches as L
import paged_reference as R

AT = L.AT


@pytest.fixture(scope="module")
def B():
    from paper_2508_16201_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding


ATTN = dict(q=AT, q_tok_stride=1792, q_head_stride=128, k_pages=AT, v_pages=AT, page_stride=16 * 512, tok_stride=512, head_stride=128, n_pages=100,
            page_size=16, page_table=AT, table_stride=50, max_pages=50, kv_lens=AT, batch=3, q_len=2, kv_len=800, n_q_heads=28, n_kv_heads=4,
            head_dim=128, softmax_scale=0.1, out=AT, workspace=AT, workspace_bytes=1 << 40)
ROPE = dict(q=AT, q_tok_stride=1792, q_head_stride=128, q_out=AT, out_tok_stride=1792, out_head_stride=128, k=AT, v=AT, kv_tok_stride=512,
            kv_head_stride=128, k_pages=AT, v_pages=AT, page_stride=16 * 512, tok_stride=512, head_stride=128, n_pages=100, page_size=16,
            page_table=AT, table_stride=50, max_pages=50, kv_lens=AT, batch=3, n_tokens=6, turns=AT, rot_dim=128, magnitude=1.0, n_q_heads=28,
            n_kv_heads=4, head_dim=128)
ASSIGN = dict(old_table=AT, old_stride=50, old_rows=3, old_max_pages=50, parent=AT, keep_len=AT, new_len=AT, batch=3, page_table=2 * AT, table_stride=50,
              max_pages=50, n_pages=100, page_size=16, copy_start=AT, copy_rows=AT, ref_counts=AT, status=AT, workspace=AT, workspace_bytes=1 << 40)
COPY = dict(k_src=AT, v_src=AT, src_layer_stride=819200, src_page_stride=8192, src_tok_stride=512, src_head_stride=128, src_pages=100, src_page_size=16,
            src_table=AT, src_table_stride=50, src_rows=3, src_max_pages=50, k_dst=2 * AT, v_dst=2 * AT, dst_layer_stride=819200, dst_page_stride=8192,
            dst_tok_stride=512, dst_head_stride=128, dst_pages=100, dst_page_size=16, dst_table=AT, dst_table_stride=50, dst_max_pages=50, n_layers=2,
            batch=3, n_rows=AT, max_rows=20, n_kv_heads=4, head_dim=128)
CALLS = {"specvlm_paged_attn": ATTN, "specvlm_rope_append": ROPE, "specvlm_pages_assign": ASSIGN, "specvlm_pages_copy": COPY}

REFUSED = [
    # (function, what is changed, status)
    *[("specvlm_paged_attn", {k: None}, -1) for k in ("q", "k_pages", "v_pages", "page_table", "kv_lens", "out")],
    *[("specvlm_paged_attn", {k: -1}, -1) for k in ("batch", "q_len", "kv_len", "n_pages", "max_pages", "window", "n_sinks", "table_stride")],
    ("specvlm_paged_attn", {"n_q_heads": 27}, -1), ("specvlm_paged_attn", {"n_kv_heads": 0}, -1), ("specvlm_paged_attn", {"page_size": 0}, -1),
    ("specvlm_paged_attn", {"softmax_scale": -1.0}, -1), ("specvlm_paged_attn", {"softmax_scale": float("nan")}, -1),
    ("specvlm_paged_attn", {"kv_len": 801}, -1), ("specvlm_paged_attn", {"kv_len": 1}, -1), ("specvlm_paged_attn", {"n_pages": 0}, -1),
    ("specvlm_paged_attn", {"head_dim": 96}, -2), ("specvlm_paged_attn", {"page_size": 24}, -2), ("specvlm_paged_attn", {"q_len": 65}, -2),
    ("specvlm_paged_attn", {"batch": (1 << 25) + 1, "q_len": 1, "kv_len": 16, "n_q_heads": 4}, -2),
    ("specvlm_paged_attn", {"page_size": 1 << 24, "kv_len": (1 << 24) * 50}, 0), ("specvlm_paged_attn", {"page_size": 1 << 26, "kv_len": (1 << 30) + 1}, -2),
    *[("specvlm_paged_attn", {k: 12}, -2) for k in ("q_tok_stride", "q_head_stride", "page_stride", "tok_stride", "head_stride")],
    *[("specvlm_paged_attn", {k: AT + 8}, -2) for k in ("q", "k_pages", "v_pages", "out")],
    ("specvlm_paged_attn", {"tok_stride": 1 << 26}, -2), ("specvlm_paged_attn", {"workspace": None}, -3),
    ("specvlm_paged_attn", {"workspace": AT + 16}, -3), ("specvlm_paged_attn", {"workspace_bytes": 1000}, -3),
    *[("specvlm_rope_append", {k: None}, -1) for k in ("q_out", "k", "v", "k_pages", "v_pages", "page_table", "kv_lens", "turns")],
    *[("specvlm_rope_append", {k: -1}, -1) for k in ("batch", "n_tokens", "n_pages", "max_pages", "rot_dim", "n_q_heads", "n_kv_heads", "table_stride")],
    ("specvlm_rope_append", {"n_tokens": 7}, -1), ("specvlm_rope_append", {"magnitude": float("inf")}, -1), ("specvlm_rope_append", {"page_size": 0}, -1),
    ("specvlm_rope_append", {"rot_dim": 144}, -1), ("specvlm_rope_append", {"rot_dim": 24}, -2), ("specvlm_rope_append", {"head_dim": 80, "rot_dim": 64}, -2),
    ("specvlm_rope_append", {"page_size": 8}, -2),
    *[("specvlm_rope_append", {k: 4}, -2) for k in ("q_tok_stride", "out_head_stride", "kv_tok_stride", "page_stride", "tok_stride", "head_stride")],
    *[("specvlm_rope_append", {k: AT + 2}, -2) for k in ("q", "q_out", "k", "v", "k_pages", "v_pages")],
    *[("specvlm_pages_assign", {k: None}, -1) for k in ("old_table", "parent", "keep_len", "new_len", "page_table", "copy_start", "copy_rows", "ref_counts", "status")],
    *[("specvlm_pages_assign", {k: -1}, -1) for k in ("old_rows", "old_max_pages", "batch", "max_pages", "n_pages", "window", "n_sinks", "old_stride")],
    ("specvlm_pages_assign", {"page_size": 0}, -1), ("specvlm_pages_assign", {"page_size": 40}, -2), ("specvlm_pages_assign", {"table_stride": 49}, -1),
    ("specvlm_pages_assign", {"workspace": None}, -3), ("specvlm_pages_assign", {"workspace_bytes": 300}, -3), ("specvlm_pages_assign", {"workspace": AT + 4}, -3),
    # the new table over the old one: the same, a row on, from behind, into the last row, one row each;  but columns of one table side by side are two
    *[("specvlm_pages_assign", {"page_table": AT + 4 * at}, -1) for at in (0, 50, 37, -149, 149)],
    ("specvlm_pages_assign", {"page_table": AT + 4 * 150}, 0), ("specvlm_pages_assign", {"page_table": AT - 4 * 150}, 0),
    ("specvlm_pages_assign", {"page_table": AT + 4 * 50, "old_stride": 100, "table_stride": 100}, 0),
    ("specvlm_pages_assign", {"page_table": AT + 4 * 49, "old_stride": 100, "table_stride": 100}, -1),
    ("specvlm_pages_assign", {"page_table": AT - 4 * 40, "old_stride": 100, "table_stride": 100}, -1),
    ("specvlm_pages_assign", {"page_table": AT + 4 * 50, "old_stride": 100, "table_stride": 101}, -1),
    ("specvlm_pages_assign", {"page_table": AT, "old_rows": 0}, 0), ("specvlm_pages_assign", {"batch": 0, "ref_counts": None}, -1),
    *[("specvlm_pages_copy", {k: None}, -1) for k in ("k_src", "k_dst", "v_src", "v_dst", "src_table", "dst_table")],
    *[("specvlm_pages_copy", {k: -1}, -1) for k in ("src_pages", "src_rows", "src_max_pages", "dst_pages", "dst_max_pages", "n_layers", "batch", "max_rows",
                                                     "src_table_stride", "dst_table_stride", "idx_stride")],
    ("specvlm_pages_copy", {"cu_idx": AT}, -1), ("specvlm_pages_copy", {"src_rows": 2}, -1), ("specvlm_pages_copy", {"n_kv_heads": 0}, -1),
    ("specvlm_pages_copy", {"head_dim": 32}, -2), ("specvlm_pages_copy", {"src_page_size": 20}, -2), ("specvlm_pages_copy", {"dst_page_size": 20}, -2),
    ("specvlm_pages_copy", {"dst_tok_stride": 20}, -2), ("specvlm_pages_copy", {"k_src": AT + 8}, -2), ("specvlm_pages_copy", {"batch": 65536, "src_rows": 65536}, -2),
    ("specvlm_pages_copy", {"n_layers": 40000}, -2), ("specvlm_pages_copy", {"max_rows": (1 << 30) + 1}, -2),
    ("specvlm_pages_copy", {"max_rows": 1 << 30}, -2), ("specvlm_pages_copy", {"max_rows": 1 << 30, "k_dst": AT, "v_dst": AT}, 0),
]
NOTHING = [("specvlm_paged_attn", {"batch": 0}), ("specvlm_paged_attn", {"q_len": 0}), ("specvlm_rope_append", {"batch": 0}), ("specvlm_rope_append", {"n_tokens": 0}),
           ("specvlm_rope_append", {"q": None, "k": None, "v": None}), ("specvlm_pages_assign", {"batch": 0, "n_pages": 0}), ("specvlm_pages_copy", {"batch": 0}),
           ("specvlm_pages_copy", {"n_layers": 0}), ("specvlm_pages_copy", {"max_rows": 0})]


def test_refusals_launch_nothing(tmp_path):
    got = L.launches([(f, {**CALLS[f], **change}) for f, change, _ in REFUSED] + [(f, {**CALLS[f], **change}) for f, change in NOTHING], tmp_path)
    for (f, change, want), (status, launched) in zip(REFUSED, got):
        assert status == want, (f, change, status)
        assert want == 0 or not launched, (f, change)
    for (f, change), (status, launched) in zip(NOTHING, got[len(REFUSED):]):
        assert status == 0 and not launched, (f, change, status, launched)


def test_launches(tmp_path):
    """One launch for the rows of a copy and for rotary positions; a launch that fails is said."""
    got = L.launches([("specvlm_rope_append", ROPE), ("specvlm_pages_copy", COPY), ("specvlm_pages_copy", {**COPY, "k_dst": AT, "v_dst": AT}),
                      ("specvlm_rope_append", {**ROPE, "q": None, "q_out": None}), ("specvlm_rope_append", {**ROPE, "k": None, "v": None})], tmp_path)
    assert [status for status, _ in got] == [0] * 5
    assert [len(launched) for _, launched in got] == [1] * 5
    (status, launched), = L.launches([("specvlm_pages_assign", {**ASSIGN, "batch": 0, "workspace": None})], tmp_path)
    assert status == 0 and len(launched) == 1                                          # no rows: nobody holds a page
    assert "true" in got[2][1][0][0] and "false" in got[1][1][0][0]                     # one pool: in order


def test_workspace_queries(B):
    need = B.paged_attn_workspace_bytes(3, 2, 28, 4, 128)
    assert need > 0
    for bad in ((3, 2, 28, 4, 96), (3, 65, 28, 4, 128), (0, 2, 28, 4, 128), (3, 2, 27, 4, 128), (-1, 2, 28, 4, 128)):
        assert B.paged_attn_workspace_bytes(*bad) == 0
    assert B.lib().specvlm_pages_assign_workspace_bytes(3, 100) > 0
    assert B.lib().specvlm_pages_assign_workspace_bytes(3, -1) == 0


def test_status_string(B):
    assert B.status_string(-5) not in (B.status_string(-99), B.status_string(-1))


@pytest.mark.parametrize("rot", [2, 16, 64, 128])
@pytest.mark.parametrize("kind", [dict(), dict(scaling="linear", factor=8.0), dict(scaling="base", factor=4.0),
                                  dict(scaling="by-parts", factor=32.0, original_len=4096), dict(scaling="by-parts", factor=1.1, original_len=100, beta_fast=3.0, beta_slow=0.5)])
def test_turns(B, rot, kind):
    if kind.get("scaling") == "base" and rot == 2:
        with pytest.raises(B.SpecVLMError):
            B.rope_turns(rot, 1e4, device="cpu", **kind)
        return
    for base in (1e4, 5e5, 1e6, 123.25):
        turns = B.rope_turns(rot, base, device="cpu", **kind).numpy().view(np.uint64)
        want = R.frequencies(rot, base, kind.get("scaling"), kind.get("factor", 1.0), kind.get("original_len", 0.0), kind.get("beta_fast", 32.0),
                             kind.get("beta_slow", 1.0)) / (2 * np.longdouble("3.14159265358979323846264338327950288"))
        # both in 64-bit mantissas: a few steps of the last bit of each
        assert (np.abs(turns.astype(np.longdouble) * np.longdouble(2.0) ** -64 - want) <= 64 * np.longdouble(2.0) ** -64 * want + np.longdouble(2.0) ** -64).all()
        assert len(turns) == rot // 2


def test_turns_of_each_kind_mean_what_they_say(B):
    plain = B.rope_turns(64, 1e4, device="cpu").numpy().astype(np.float64)
    assert np.allclose(B.rope_turns(64, 1e4, scaling="linear", factor=4, device="cpu").numpy(), plain / 4, rtol=1e-12)
    base = B.rope_turns(64, 1e4, scaling="base", factor=4, device="cpu").numpy()
    assert np.isclose(base[0], plain[0], rtol=1e-12) and np.isclose(base[-1], plain[-1] / 4, rtol=1e-12)
    parts = B.rope_turns(64, 1e4, scaling="by-parts", factor=4, original_len=4096, device="cpu").numpy() / plain
    assert np.isclose(parts[0], 1, rtol=1e-12) and np.isclose(parts[-1], 0.25, rtol=1e-12) and (np.diff(parts) <= 1e-12).all()


def test_turns_refused(B):
    for kw in (dict(rot_dim=15), dict(rot_dim=-2), dict(base=0.0), dict(base=float("nan")), dict(scaling="linear", factor=0.5), dict(scaling="base", factor=float("inf")),
               dict(scaling="by-parts", factor=2.0), dict(scaling="by-parts", factor=2.0, original_len=100, beta_fast=1.0, beta_slow=1.0)):
        args = {"rot_dim": 64, "base": 1e4, **kw}
        with pytest.raises(B.SpecVLMError):
            B.rope_turns(args.pop("rot_dim"), args.pop("base"), device="cpu", **args)
    assert B.lib().specvlm_rope_turns(64, None, None) == -1
    assert len(B.rope_turns(0, 1e4, device="cpu")) == 0


def test_the_plain_implementations_agree_with_the_oracle(oracle_lib):
    """paged_reference's attention over pages in order is the oracle's over the same rows, chain and tree."""
    rng = np.random.default_rng(1)
    from paper_2508_16201_amd import synth
    q, k, v = (synth.f32_to_bf16_bits(rng.standard_normal(s).astype(np.float32)) for s in ((5, 4, 64), (48, 2, 64), (48, 2, 64)))
    table = np.arange(3, dtype=np.int32)[None]
    pages = [R.values(x).reshape(3, 16, 2, 64) for x in (k, v)]
    masks = np.asarray(synth.ancestor_masks(synth.make_tree(5, 3))).astype(np.uint64)
    for m in (None, masks):
        out, lse, _, _, _ = R.paged_attention(R.values(q), *pages, table, [40], [5], 0.125, masks=m)
        want, want_lse = oracle_lib.decode_attn(q, k[:40], v[:40], 0.125) if m is None else oracle_lib.tree_attn(q, k[:40], v[:40], m, 0.125)
        assert np.allclose(out, want, atol=1e-12) and np.allclose(lse, want_lse, atol=1e-12)


def test_the_binding_refuses_tensors_off_the_gpu(B):
    import torch
    k, v = (torch.zeros(4, 16, 2, 64).bfloat16() for _ in range(2))
    i = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: B.paged_attn(torch.zeros(1, 4, 64).bfloat16(), k, v, i[None], i, 0.1),
                 lambda: B.rope_append(torch.zeros(1, 2, 64).bfloat16(), torch.zeros(1, 2, 64).bfloat16(), k, v, i[None], i),
                 lambda: B.pages_assign(i[None], i, i, i, 4, 16),
                 lambda: B.pages_copy(k[None], v[None], i[None], k[None], v[None], i[None], i, 1)):
        with pytest.raises(ValueError):
            call()
