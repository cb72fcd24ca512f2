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


LIMITS = [
    # (function, arguments, the one that grows, its largest value): a launch has fewer than 2^32 threads
    ("specvlm_paged_attn", {**ATTN, "kv_len": 16, "q_len": 1, "n_q_heads": 1, "n_kv_heads": 1, "out": 2 * AT}, "batch", (2 ** 32 - 1) // 384),
    ("specvlm_paged_attn", {**ATTN, "kv_len": 16, "q_len": 1, "n_q_heads": 8, "n_kv_heads": 8, "head_dim": 64, "out": 2 * AT}, "batch", (2 ** 32 - 1) // 512 // 8),
    ("specvlm_paged_attn", {**ATTN, "kv_len": 2000, "page_size": 160, "q_len": 1, "n_q_heads": 1, "n_kv_heads": 1, "out": 2 * AT}, "batch", 2 ** 24 - 1),
    ("specvlm_paged_attn", {**ATTN, "kv_len": 2000, "page_size": 160, "q_len": 1, "n_q_heads": 5, "n_kv_heads": 1, "out": 2 * AT}, "batch", 2 ** 23 - 1),
    ("specvlm_rope_append", {**ROPE, "batch": 1}, "n_tokens", 2 ** 26 - 4),
    ("specvlm_pages_assign", {**ASSIGN, "old_rows": 0}, "batch", 2 ** 24 - 2),
    ("specvlm_pages_assign", {**ASSIGN, "old_rows": 0, "max_pages": 60, "table_stride": 60, "n_pages": 1 << 20}, "batch", 2 ** 24 - 1 - 1024),
    ("specvlm_pages_assign", {**ASSIGN, "old_max_pages": 600, "max_pages": 30, "old_stride": 600, "page_table": 4 * AT}, "batch", (2 ** 24 - 2) // 3),
]


@pytest.mark.parametrize("case", range(len(LIMITS)))
def test_the_largest_launches(tmp_path, case):
    """What would be a larger launch is refused before any other, and the largest are what they may be."""
    function, args, grows, most = LIMITS[case]
    (status, launched), (refused, none) = L.launches([(function, {**args, grows: most}), (function, {**args, grows: most + 1})], tmp_path)
    assert status == 0
    for kernel, grid, block, *_ in launched:
        assert all(g * b < 2 ** 32 for g, b in zip(grid, block)), (kernel, grid, block)
    assert refused == -2 and not none
