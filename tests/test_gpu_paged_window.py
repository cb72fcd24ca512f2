"""specvlm_paged_attn with windows as long as their type has, over blocks whose masks name later places too."""
import numpy as np
import pytest
import torch

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


@pytest.mark.parametrize("heads", [(4, 1, 64), (8, 2, 128)])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 40, 8192, 100, 64])
def test_windows_longer_than_the_cache(B, heads, window):
    """Every node of the block sees every other, before it and behind it: no window as long as the cache hides one."""
    kv_lens, q_lens = [64, 100], [64, 64]
    q, k, v, table = build(51, kv_lens, q_lens, heads, 16)
    masks = np.full(128, 2 ** 64 - 1, dtype=np.uint64)
    want, want_lse, tol, tol_lse, _ = R.paged_attention(R.values(q), R.values(k), R.values(v), table, kv_lens, q_lens, 0.1, window, 0, masks)
    mask = torch.from_numpy(masks.view(np.int64)).cuda()
    for name, (entries, lens, how) in variants(table, kv_lens, q_lens, 16).items():
        got, lse = B.paged_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), i32(entries), i32(lens), 0.1, window=window, ancestor_mask=mask, want_lse=True, **how)
        assert (np.abs(host_f64(got) - want) <= tol).all(), name
        assert (np.abs(host_f64(lse) - want_lse) <= tol_lse).all(), name
