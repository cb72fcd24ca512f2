"""specvlm_shared_attn and specvlm_cross_attn with offsets, lengths and groups of which some or all say nothing that fits together."""
import numpy as np
import pytest
import torch

import shared_reference as S
from gpu_util import dev_bf16, host_f64, rnd_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2508_16201_amd import binding
    binding.lib()
    return binding


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def shared(B, q, pages, table, kv_lens, groups, cu_q, q_len, kv_len, scale=0.125):
    """K and V in the same pages -> (out, lse), where nothing is written 7."""
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    batch, (tq, hq, d), (n_pages, ps, hkv, _) = len(kv_lens), q.shape, pages.shape
    ws = B.new_workspace(B.shared_attn_workspace_bytes(batch, tq, hq, hkv, d), q.device)
    rc = B.lib().specvlm_shared_attn(q.data_ptr(), q.stride(0), q.stride(1), pages.data_ptr(), pages.data_ptr(), pages.stride(0), pages.stride(1), pages.stride(2),
                                     n_pages, ps, table.data_ptr(), table.stride(0), table.shape[1], kv_lens.data_ptr(), groups.data_ptr(), cu_q.data_ptr(), batch,
                                     tq, q_len, kv_len, hq, hkv, d, scale, None, out.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(),
                                     torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    torch.cuda.synchronize()
    return out, lse


def cross(B, q, k, cu_q, cu_kv, ranges=None, scale=0.125):
    """K and V the same -> (out, lse), where nothing is written 7."""
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    batch, (tq, hq, d), (tk, hkv, _) = len(cu_q) - 1, q.shape, k.shape
    ws = B.new_workspace(B.cross_attn_workspace_bytes(batch, tq, hq, hkv, d), q.device)
    rc = B.lib().specvlm_cross_attn(q.data_ptr(), q.stride(0), q.stride(1), k.data_ptr(), k.data_ptr(), k.stride(0), k.stride(1), cu_q.data_ptr(), cu_kv.data_ptr(),
                                    batch, tq, tk, hq, hkv, d, scale, None if ranges is None else ranges.data_ptr(), out.data_ptr(), lse.data_ptr(), ws.data_ptr(),
                                    ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("batch", [256, 257, 600])
@pytest.mark.parametrize("what", ["no tokens", "shorter than their blocks", "longer than the call says", "empty blocks"])
def test_a_batch_of_skipped_requests_writes_nothing(B, batch, what):
    """Up to 1200 entries, none of which has work (slots of a service that are all idle)."""
    q, pages = dev_bf16(rnd_bits((2 * batch, 4, 64), 1)), dev_bf16(rnd_bits((8, 16, 1, 64), 2))
    lens = {"no tokens": 0, "shorter than their blocks": 1, "longer than the call says": 97, "empty blocks": 60}[what]
    cu_q = torch.zeros(batch + 1, dtype=torch.int32, device="cuda") if what == "empty blocks" else i32(2 * np.arange(batch + 1))
    out, lse = shared(B, q, pages, torch.zeros((batch, 8), dtype=torch.int32, device="cuda"), torch.full((batch,), lens, dtype=torch.int32, device="cuda"),
                      torch.zeros((3, batch), dtype=torch.int32, device="cuda"), cu_q, 2, 96)
    assert (out == 7.0).all() and (lse == 7.0).all()


@pytest.mark.parametrize("batch", [512, 513, 1500])
@pytest.mark.parametrize("ranges", [False, True])
def test_a_batch_of_empty_entries_writes_nothing(B, batch, ranges):
    q, k = dev_bf16(rnd_bits((70, 4, 64), 1)), dev_bf16(rnd_bits((100, 1, 64), 2))
    seen = i32([[0, 100]] * 70) if ranges else None
    for first in (0, 70, 1 << 20):
        cu_q = torch.full((batch + 1,), first, dtype=torch.int32, device="cuda")
        out, lse = cross(B, q, k, cu_q, i32([0] * batch + [100]), seen)
        assert (out == 7.0).all() and (lse == 7.0).all()


def test_work_behind_many_entries_that_have_none(B):
    """1100 empty entries, then one."""
    q, k = rnd_bits((3, 4, 64), 5), rnd_bits((200, 1, 64), 6)
    want, want_lse, tol, tol_lse = S.cross_attention(S.values(q), S.values(k), S.values(k), [3], [200], 0.125)
    out, lse = cross(B, dev_bf16(q), dev_bf16(k), i32([0] * 1101 + [3]), i32([0] * 1101 + [200]))
    assert (np.abs(host_f64(out) - want) <= tol).all() and (np.abs(lse.double().cpu().numpy() - want_lse) <= tol_lse).all()


@pytest.mark.parametrize("cu_q,q_len,left", [([0, 5, 100, 20], 95, [0, 1]), ([50, 60, 10, 40, 45], 50, [0, 2, 3]), ([50, 60, 10, 40, 90], 30, [0, 2]),
                                             ([10, 12, 0, 8, -5, 14], 20, [0, 2]), ([0, 5, 300, 9, 20], 20, [0, 3])])
@pytest.mark.parametrize("shared_tokens", [0, 96])
def test_requests_of_a_group_whose_queries_lie_elsewhere(B, cu_q, q_len, left, shared_tokens):
    """Offsets that descend inside a group: who has no queries is skipped, whose queries are not among the group's is taken alone."""
    batch, hq, d, n_queries, kv_len, ps = len(cu_q) - 1, 14, 64, 100, 700, 16
    q, k = rnd_bits((n_queries, hq, d), 31), rnd_bits((batch * kv_len // ps + batch, ps, 2, d), 32)
    width = -(-kv_len // ps)
    table = np.arange(batch * width, dtype=np.int32).reshape(batch, width) % len(k)
    table[:, :shared_tokens // ps] = table[0, :shared_tokens // ps]
    groups = np.zeros((3, batch), dtype=np.int32)
    groups[1, 0], groups[2] = batch, shared_tokens
    out, lse = shared(B, dev_bf16(q), dev_bf16(k), i32(table), i32([kv_len] * batch), i32(groups), i32(cu_q), q_len, kv_len)
    got, got_lse, written = host_f64(out), lse.double().cpu().numpy(), np.zeros(n_queries, dtype=bool)
    for b in left:
        rows = slice(cu_q[b], cu_q[b + 1])
        x = S.values(k)[table[b]].reshape(-1, 2, d)[:kv_len]
        want, want_lse, tol, tol_lse = S.all_heads(S.values(q[rows]), x, x, 0.125, S.block_sees(kv_len, cu_q[b + 1] - cu_q[b]))
        assert (np.abs(got[rows] - want) <= tol).all() and (np.abs(got_lse[rows] - want_lse) <= tol_lse).all()
        written[rows] = True
    assert (got[~written] == 7.0).all() and (got_lse[~written] == 7.0).all()


@pytest.mark.parametrize("length", [-2 ** 31, -2 ** 31 + 1, -1, 0, 2 ** 31 - 1])
@pytest.mark.parametrize("tokens", [32, 1 << 20, 2 ** 31 - 16])
def test_a_first_request_of_no_possible_length_has_no_group(B, length, tokens):
    q, k = rnd_bits((6, 4, 64), 41), rnd_bits((20, 16, 1, 64), 42)
    table = np.arange(15, dtype=np.int32).reshape(3, 5) + 2
    groups = np.array([[0, 0, 0], [3, 0, 0], [tokens] * 3], dtype=np.int32)
    out, lse = shared(B, dev_bf16(q), dev_bf16(k), i32(table), i32([length, 70, 33]), i32(groups), i32([0, 2, 4, 6]), 2, 80)
    got, got_lse = host_f64(out), lse.double().cpu().numpy()
    assert (got[:2] == 7.0).all() and (got_lse[:2] == 7.0).all()
    for b, n in ((1, 70), (2, 33)):
        rows, x = slice(2 * b, 2 * b + 2), S.values(k)[table[b]].reshape(-1, 1, 64)[:n]
        want, want_lse, tol, tol_lse = S.all_heads(S.values(q[rows]), x, x, 0.125, S.block_sees(n, 2))
        assert (np.abs(got[rows] - want) <= tol).all() and (np.abs(got_lse[rows] - want_lse) <= tol_lse).all()


def entries_in_order(order, lens, gap=0):
    """cu_q in which the entries of these lengths lie in another order than their numbers have, with skipped ones in between -> (cu_q, numbers, begins)."""
    begins = np.zeros(len(lens), dtype=int)
    begins[order] = np.concatenate([[0], np.cumsum(np.asarray(lens)[order] + gap)[:-1]])
    cu_q, numbers = [], []
    for begin, n in zip(begins, lens):
        if not cu_q or cu_q[-1] != begin:
            assert not cu_q or cu_q[-1] > begin, "an entry in front of this one would have queries"
            cu_q.append(int(begin))
        numbers.append(len(cu_q) - 1)
        cu_q.append(int(begin + n))
    return cu_q, numbers, begins


@pytest.mark.parametrize("heads", [(8, 1, 64), (28, 4, 128)])
@pytest.mark.parametrize("lens", [[64, 32], [5, 40, 33], [70, 1, 32, 90], [3] * 90])
@pytest.mark.parametrize("kind", ["cross", "ranges", "paged"])
def test_entries_whose_queries_lie_in_descending_order(B, heads, lens, kind):
    """The first entry's queries behind the second one's, and so on: a descending entry, which is skipped, between each two."""
    hq, hkv, d = heads
    cu_q, numbers, begins = entries_in_order(np.arange(len(lens))[::-1], lens)
    n_queries, batch, states = sum(lens), len(cu_q) - 1, 160
    if lens == [64, 32]:
        assert cu_q == [32, 96, 0, 32]
    q, k = rnd_bits((n_queries, hq, d), 51), rnd_bits((batch * states, hkv, d), 52)
    at = np.random.default_rng(53).integers(-9, states + 20, (n_queries, 2)).astype(np.int32)
    ranges = np.sort(at, axis=1) if kind == "ranges" else None
    if kind == "paged":
        out, lse = shared(B, dev_bf16(q), dev_bf16(k.reshape(-1, 16, hkv, d)), i32(np.arange(batch * 10).reshape(batch, 10)), i32([states] * batch),
                          torch.zeros((3, batch), dtype=torch.int32, device="cuda"), i32(cu_q), max(lens), states)
    else:
        out, lse = cross(B, dev_bf16(q), dev_bf16(k), i32(cu_q), i32(np.arange(batch + 1) * states), None if ranges is None else i32(ranges))
    got, got_lse = host_f64(out), lse.double().cpu().numpy()
    for e, begin, n in zip(numbers, begins, lens):
        rows, x = slice(begin, begin + n), S.values(k)[e * states:(e + 1) * states]
        if kind == "paged":
            want, want_lse, tol, tol_lse = S.all_heads(S.values(q[rows]), x, x, 0.125, S.block_sees(states, n))
        else:
            want, want_lse, tol, tol_lse = S.cross_attention(S.values(q[rows]), x, x, [n], [states], 0.125, None if ranges is None else ranges[rows])
        some = np.isfinite(want_lse)
        assert (np.abs(got[rows] - want) <= tol).all()
        assert (got_lse[rows][~some] == -np.inf).all() and (np.abs(got_lse[rows][some] - want_lse[some]) <= tol_lse[some]).all()


def test_ranges_of_entries_that_have_each_query_many_times(B):
    """More shares than there are numbers for, and their sum more than an int holds: nothing is written, and the next call is as ever."""
    n_queries = 4096
    q, k = rnd_bits((n_queries + 9, 64, 64), 1), rnd_bits((64, 1, 64), 2)
    seen = i32(np.tile([[0, 64]], (n_queries + 9, 1)))
    cu = torch.zeros(8193, dtype=torch.int32, device="cuda")
    cu[1::2] = n_queries
    out, lse = cross(B, dev_bf16(q), dev_bf16(k), cu, torch.clamp(cu, max=64), seen)
    assert (out == 7.0).all() and (lse == 7.0).all()
    want, want_lse, tol, tol_lse = S.cross_attention(S.values(q), S.values(k), S.values(k), [n_queries + 9], [64], 0.125)
    out, lse = cross(B, dev_bf16(q), dev_bf16(k), i32([0, n_queries + 9]), i32([0, 64]), seen)
    assert (np.abs(host_f64(out) - want) <= tol).all() and (np.abs(lse.double().cpu().numpy() - want_lse) <= tol_lse).all()
