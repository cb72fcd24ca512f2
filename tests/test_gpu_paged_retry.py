"""Forks that find too few pages: what the rows are left with, and both ways on from there."""
import numpy as np
import pytest
import torch

from gpu_util import dev_bf16, rnd_bits
from test_gpu_paged_attn import i32

pytestmark = pytest.mark.gpu
PS, KEPT, HEADS, D = 16, 24, 2, 64


@pytest.fixture(scope="module")
def B():
    from paper_2508_16201_amd import binding
    binding.lib()
    return binding


class Pool:
    """One request of 24 tokens in pages 0 and 1 of three, the third with rows that nobody wrote; a reference of its keys in order."""

    def __init__(self, B):
        self.B = B
        self.k, self.v = (torch.full((1, 3, PS, HEADS, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.rows = [dev_bf16(rnd_bits((KEPT + 1, HEADS, D), i)) for i in (1, 2)]
        for pool, rows in zip((self.k, self.v), self.rows):
            pool[0, 0], pool[0, 1, :KEPT - PS] = rows[:PS], rows[PS:KEPT]
        self.table = i32([[0, 1]])
        self.q = dev_bf16(rnd_bits((1, 4, D), 3))

    def assign(self, table, parent, keep, new):
        got = self.B.pages_assign(table, i32(parent), i32(keep), i32(new), 3, PS)
        return got[0], got[1], got[2], got[4].tolist()

    def copy(self, old, table, parent, start, rows):
        self.B.pages_copy(self.k, self.v, old, self.k, self.v, table, rows, PS, src_row=i32(parent), src_start=start, dst_start=start)

    def append(self, table, lens):
        """The token behind the kept ones, the same for every row."""
        n = table.shape[0]
        k, v = (r[KEPT:].expand(n, HEADS, D).contiguous() for r in self.rows)
        self.B.rope_append(k, v, self.k[0], self.v[0], table, i32(lens))

    def sees(self, table, n, rows):
        """Each row's attention is that over the tokens in order."""
        want = self.B.decode_attn(self.q, self.rows[0][:n], self.rows[1][:n], 0.125)
        got = self.B.paged_attn(self.q.repeat(table.shape[0], 1, 1), self.k[0], self.v[0], table, i32([n] * table.shape[0]), 0.125)
        off = (got.float() - want.float()).abs().amax((1, 2)).tolist()
        # (both round to bf16, decode_attn its probabilities and parts too: 2^-8 each of values below 5)
        return all((off[b] <= 3 * 2.0 ** -8 * 5) == (b in rows) for b in range(table.shape[0]))


def short_of_pages(B):
    p = Pool(B)
    first, start, rows, status = p.assign(p.table, [0, 0, 0], [KEPT] * 3, [KEPT + 1] * 3)
    assert status == [0, 0, -5]
    assert first.tolist() == [[0, 1], [0, 2], [0, -1]] and rows.tolist() == [0, KEPT - PS, 0]
    assert p.table.tolist() == [[0, 1]]
    return p, first, start, rows


def test_the_assignment_is_made_again_from_the_old_table(B):
    p, *_ = short_of_pages(B)
    table, start, rows, status = p.assign(p.table, [0, 0], [KEPT] * 2, [KEPT + 1] * 2)
    assert status == [0, 0] and table.tolist() == [[0, 1], [0, 2]]
    p.copy(p.table, table, [0, 0], start, rows)
    p.append(table, [KEPT + 1] * 2)
    assert p.sees(table, KEPT + 1, {0, 1})


def test_the_row_goes_on_later_from_its_whole_pages(B):
    p, first, start, rows = short_of_pages(B)
    p.copy(p.table, first, [0, 0, 0], start, rows)
    p.append(first, [KEPT + 1, KEPT + 1, 0])
    assert p.sees(first[:2], KEPT + 1, {0, 1})
    # the second row ends, and its page goes to the third, which writes what it had lost
    p.k[0, 2], p.v[0, 2] = float("nan"), float("nan")
    table, start, rows, status = p.assign(first, [0, 2], [KEPT + 1, PS], [KEPT + 1, KEPT + 1])
    assert status == [0, 0] and table.tolist() == [[0, 1], [0, 2]] and rows.tolist() == [0, 0]
    p.copy(first, table, [0, 0], i32([PS, PS]), i32([0, KEPT + 1 - PS]))
    assert p.sees(table, KEPT + 1, {0, 1})


def test_a_page_that_is_none_where_the_kept_tokens_end(B):
    """Kept all the same it is a page of the row's, with nothing to copy: the caller's rows are to be written."""
    p, first, _, _ = short_of_pages(B)
    table, start, rows, status = p.assign(first, [0, 2], [KEPT, KEPT], [KEPT + 1] * 2)
    assert status == [0, 0] and table.tolist() == [[0, 1], [0, 2]] and rows.tolist() == [0, 0]
    p.copy(first, table, [0, 0], i32([PS, PS]), i32([0, KEPT - PS]))
    p.append(table, [KEPT + 1] * 2)
    assert p.sees(table, KEPT + 1, {0, 1})
