"""The native marshalling of pages_shared, shared_attn and cross_attn against the general code of binding.py."""
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


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("given", [False, True])
def test_shared_attn(monkeypatch, ragged, given):
    k, v = bf16(9, 16, 2, 64), bf16(9, 16, 2, 64, seed=2)
    q, table, lens, groups = bf16(6, 8, 64, seed=3), i32(4, 7, 1, 0, 4, 7, 2, 3).view(2, 4), i32(40, 64), i32(0, 0, 2, 0, 32, 32).view(3, 2)
    more = dict(cu_q=i32(0, 2, 6), max_q_len=4, max_kv_len=64) if ragged else dict(ancestor_mask=torch.full((6,), 7, device="cuda"))
    if given:
        more.update(out=torch.zeros_like(q), workspace=B.new_workspace(B.shared_attn_workspace_bytes(2, 6, 8, 2, 64)))
    for lse in (False, True):
        a, b = both(monkeypatch, lambda: B.shared_attn(q, k, v, table, lens, 0.125, groups, want_lse=lse, **more))
        same(a, b)
        if given:
            assert (a[0] if lse else a) is more["out"]


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("given", [False, True])
def test_cross_attn(monkeypatch, ragged, given):
    q, k, v = bf16(6, 8, 64), bf16(70, 2, 64, seed=2), bf16(70, 2, 64, seed=3)
    more = dict(cu_q=i32(0, 2, 6), cu_kv=i32(0, 0, 70)) if ragged else dict(key_ranges=i32(0, 70, 3, 9, 5, 5, 60, 99, -4, 40, 1, 2).view(6, 2))
    if given:
        more.update(out=torch.zeros_like(q), workspace=B.new_workspace(B.cross_attn_workspace_bytes(2, 6, 8, 2, 64)))
    for lse in (False, True):
        a, b = both(monkeypatch, lambda: B.cross_attn(q, k, v, 0.125, want_lse=lse, **more))
        same(a, b)
        if given:
            assert (a[0] if lse else a) is more["out"]


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("given", [False, True])
def test_pages_shared(monkeypatch, ragged, given):
    table, lens = i32(4, 7, 1, 0, 4, 7, 2, 3, 4, 7, 2, 5).view(3, 4), i32(40, 64, 64)
    more = dict(cu_q=i32(0, 2, 6, 7)) if ragged else {}
    if given:
        more.update(groups=torch.zeros((3, 3), dtype=torch.int32, device="cuda"), workspace=B.new_workspace(B.pages_shared_workspace_bytes(3)))
    a, b = both(monkeypatch, lambda: B.pages_shared(table, lens, 9, 16, 4, min_tokens=16, **more))
    same(a, b)
    if given:
        assert a is more["groups"]


def test_refusals_are_the_same(monkeypatch):
    q, k, lens = bf16(6, 8, 64), bf16(9, 16, 2, 64), i32(40, 64)
    table, groups = i32(4, 7, 1, 0, 4, 7, 2, 3).view(2, 4), i32(0, 0, 2, 0, 32, 32).view(3, 2)
    calls = [lambda: B.shared_attn(q, k, k, table, lens, 0.125, groups[:2]), lambda: B.shared_attn(q[:5], k, k, table, lens, 0.125, groups),
             lambda: B.shared_attn(q, k, k[:8], table, lens, 0.125, groups), lambda: B.shared_attn(q.float(), k, k, table, lens, 0.125, groups),
             lambda: B.cross_attn(q, k, k, 0.125), lambda: B.cross_attn(q[:, :7], k[0], k[0], 0.125),
             lambda: B.cross_attn(q, k[0], k[0], 0.125, key_ranges=i32(0, 4)), lambda: B.pages_shared(table, lens.long(), 9, 16, 3),
             lambda: B.shared_attn(q, k, k, table, lens, 0.125, groups, workspace=torch.zeros(3, dtype=torch.uint8, device="cuda"))]

    def answer(call):
        try:
            call()
        except Exception as e:
            return type(e), str(e)
        return None

    for call in calls:
        a = answer(call)
        with monkeypatch.context() as m:
            m.setattr(B, "_calls", B._NoCalls())
            assert answer(call) == a is not None
