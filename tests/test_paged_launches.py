"""What the paged operators launch, seen from the host.  No GPU is touched."""
import pytest

import launches as L
from test_paged_abi import ASSIGN, ATTN, ROPE

AT = L.AT
# sizes that each of the attention's ways to a result takes
WAYS = {"slices": dict(batch=1, q_len=1, kv_len=500, n_q_heads=14, n_kv_heads=2, head_dim=64),
        "whole": dict(batch=64, q_len=1, kv_len=500, n_q_heads=14, n_kv_heads=2, head_dim=64),
        "shared": dict(batch=1, q_len=6, kv_len=8000, page_size=160, n_q_heads=64, n_kv_heads=8, head_dim=128)}


def test_the_attentions_ways(tmp_path):
    got = L.launches([("specvlm_paged_attn", {**ATTN, "out": 2 * AT, **more}) for more in WAYS.values()], tmp_path)
    assert [status for status, _ in got] == [0] * 3
    assert [[kernel.split("<")[0] for kernel, *_ in launched] for _, launched in got] == [
        ["paged_short_kernel"], ["paged_split_kernel"], ["paged_split_kernel", "paged_join_kernel"]]


@pytest.mark.parametrize("way", WAYS)
def test_an_output_over_the_queries_is_not_written_in_slices(tmp_path, way):
    """Each of the slices reads whole query rows, and would write a part of them while the others read."""
    (status, launched), = L.launches([("specvlm_paged_attn", {**ATTN, **WAYS[way], "out": ATTN["q"]})], tmp_path)
    assert status == 0 and launched
    assert not any("paged_short" in kernel for kernel, *_ in launched)
