"""Sizes of shared and cross attention far beyond what they serve: refused, whatever their products are.  No GPU is touched."""
import launches as L
import pytest

import test_shared_abi as T

FAR = [(batch, heads) for batch in ((1 << 31) - 1, 2029870315, 1 << 30, 1 << 24) for heads in ((1 << 29) - 1, 1 << 28, 1 << 27, 1 << 22)]


def calls():
    for batch, heads in FAR:
        for keys in (1 << 4, 545918790, 556926567, 1008403731, 1 << 30):
            many = {"cu_q": L.AT, "batch": batch, "n_queries": 1, "n_q_heads": heads, "n_kv_heads": heads}
            yield "specvlm_shared_attn", {**T.ATTN, **many, "q_len": 1, "kv_len": keys, "page_size": 1 << 30, "max_pages": 1}
            yield "specvlm_cross_attn", {**T.CROSS, **many, "n_states": keys}
            yield "specvlm_cross_attn", {**T.CROSS, **many, "n_states": keys, "key_ranges": L.AT}


def test_sizes_whose_products_wrap_are_refused(tmp_path):
    every = list(calls())
    for (f, args), (status, launched) in zip(every, L.launches(every, tmp_path)):
        assert status == -2 and not launched, (f, {k: args[k] for k in ("batch", "n_kv_heads")}, status, launched)


@pytest.mark.parametrize("batch,heads", FAR)
def test_workspaces_of_what_is_refused_are_none(batch, heads):
    from paper_2508_16201_amd import binding as B
    assert B.shared_attn_workspace_bytes(batch, 1, heads, heads, 128) == 0
    assert B.cross_attn_workspace_bytes(batch, 1, heads, heads, 128) == 0
    for n in (1 << 29, (1 << 31) - 1):
        assert B.shared_attn_workspace_bytes(1, n, 28, 4, 128) == 0 and B.cross_attn_workspace_bytes(1, n, 28, 4, 128) == 0
