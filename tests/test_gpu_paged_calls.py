"""The native marshalling of the paged functions against the general code of binding.py."""
import os

import pytest
import torch

from paper_2508_16201_amd import binding as B, build
from test_gpu_calls import bf16, both, i32, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(B.LIB_PATH) or not os.path.exists(build.CALLS):
        build.build()


def cache(batch=2, pages=9, ps=16, heads=2, d=64):
    table = torch.stack([torch.randperm(pages, device="cuda")[:4] for _ in range(batch)]).to(torch.int32)
    return bf16(pages, ps, heads, d), bf16(pages, ps, heads, d, seed=2), table


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("given", [False, True])
def test_paged_attn(monkeypatch, ragged, given):
    k, v, table = cache()
    q, lens = bf16(6, 8, 64, seed=3), i32(40, 64)
    more = dict(cu_q=i32(0, 2, 6), max_q_len=4, max_kv_len=64) if ragged else dict(window=20, n_sinks=3, ancestor_mask=torch.full((6,), 7, device="cuda"))
    if given:
        more.update(out=torch.zeros_like(q), workspace=B.new_workspace(B.paged_attn_workspace_bytes(2, 4, 8, 2, 64)))
    for lse in (False, True):
        a, b = both(monkeypatch, lambda: B.paged_attn(q, k, v, table, lens, 0.125, want_lse=lse, **more))
        same(a, b)
        if given:
            assert (a[0] if lse else a) is more["out"]


@pytest.mark.parametrize("given", [False, True])
def test_rope_append(monkeypatch, given):
    k, v, table = cache()
    q, kn, vn = bf16(6, 8, 64, seed=3), bf16(6, 2, 64, seed=4), bf16(6, 2, 64, seed=5)
    more = dict(q_out=torch.zeros_like(q), positions=i32(5, 4, 3, 2, 1, 0), cu_q=i32(0, 2, 6), interleaved=True, magnitude=1.5) if given else {}

    def call():
        pools = k.clone(), v.clone()
        got = B.rope_append(kn, vn, *pools, table, i32(40, 64), q=q, turns=B.rope_turns(32, 1e4), **more)
        return got.clone(), *pools

    same(*both(monkeypatch, call))

    def keys_alone():
        pools = k.clone(), v.clone()
        assert B.rope_append(kn, vn, *pools, table, i32(40, 64)) is None
        return pools

    same(*both(monkeypatch, keys_alone))


@pytest.mark.parametrize("given", [False, True])
def test_pages_assign(monkeypatch, given):
    table = i32(3, 1, 4, -1, 0, 2, -1, -1).view(2, 4)
    more = dict(out=torch.zeros((3, 6), dtype=torch.int32, device="cuda"), window=20, n_sinks=1,
                workspace=B.new_workspace(B.lib().specvlm_pages_assign_workspace_bytes(3, 12))) if given else {}
    a, b = both(monkeypatch, lambda: B.pages_assign(table, i32(0, 0, 1), i32(40, 40, 20), i32(50, 41, 60), 12, 16, **more))
    same(a, b)
    if given:
        assert a[0] is more["out"]


@pytest.mark.parametrize("what", ["rows", "lists", "cut", "forked"])
def test_pages_copy(monkeypatch, what):
    src, dst = bf16(3, 9, 16, 2, 64), bf16(3, 7, 32, 2, 64, seed=2)
    more = {"rows": dict(src_start=i32(1, 2)), "lists": dict(row_idx=i32(3, 5, 7, 0, 2, -1).view(2, 3), dst_start=i32(4, 5)),
            "cut": dict(row_idx=i32(3, 5, 7, 0, 2), cu_idx=i32(0, 3, 5)), "forked": dict(src_row=i32(1, 0))}[what]

    def call():
        pools = dst.clone(), dst.clone()
        B.pages_copy(src, src, i32(0, 1, 2, 3).view(2, 2), *pools, i32(5, 6).view(2, 1), None if what == "cut" else i32(3, 2), 3, **more)
        return pools

    same(*both(monkeypatch, call))


def test_refusals_are_the_general_ones():
    """What does not fit is left to the general code, and a status comes back as its error."""
    k, v, table = cache()
    q = bf16(2, 8, 64)
    with pytest.raises(ValueError):
        B.paged_attn(q, k, v, table.long(), i32(40, 64), 0.125)
    with pytest.raises(ValueError):
        B.paged_attn(q, k, v, table, i32(40, 64, 1), 0.125)
    with pytest.raises(B.SpecVLMError) as e:
        B.paged_attn(q, k, v, table, i32(40, 64), 0.125, window=-2)
    assert e.value.status == -1 and "specvlm_paged_attn" in str(e.value)
    with pytest.raises(B.SpecVLMError) as e:
        B.pages_assign(table, i32(0, 1), i32(0, 0), i32(1, 1), 9, 24)
    assert e.value.status == -2
