"""The paged cache's operators (vla_cache.h) at their edges: infinite and NaN values, many heads without keys, the most
environments, appends against the oracle's.  References and tolerances are those of test_gpu_cache.py."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2505_18719_amd import vla
from test_gpu_cache import BF, FP, PAGE, attn_tol, check_attention, f64, i32, make_cache, rand

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ environments without keys
@pytest.mark.parametrize("H,K,hd", [(320, 8, 64), (257, 1, 128), (1024, 1024, 64)])
def test_lse_of_every_head_of_environments_without_keys(H, K, hd):
    """More heads than a workgroup has threads, keys split: each head's log-sum-exp is -inf for length 0, else NaN."""
    kp, vp, table, lens = make_cache([300, 0, 40, 33, 7], K, hd, BF, 1, extra_cols=80)
    lens = np.array(lens)
    lens[2], lens[3] = -1, table.shape[1] * PAGE + 1
    q, out = rand((5, H, hd), BF, 2), torch.full((5, H, hd), 7.0, dtype=BF, device="cuda")
    lse = torch.full((5, H), 7.0, device="cuda")
    vla.paged_attention(q, kp, vp, i32(table), i32(lens), hd ** -0.5, out=out, lse=lse)
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()
    assert out[2:4].isnan().all() and lse[2:4].isnan().all()
    check_attention(out, lse, q, kp, vp, table, lens, hd ** -0.5, envs=[0, 4])


def test_lse_of_every_head_without_a_pool():
    q, lse = rand((3, 1024, 64), BF, 2), torch.full((3, 1024), 7.0, device="cuda")
    kp = torch.empty(0, 2, PAGE, 64, dtype=BF, device="cuda")
    vp = torch.empty(0, 2, 64, PAGE, dtype=BF, device="cuda")
    got = vla.paged_attention(q, kp, vp, torch.zeros(3, 99, dtype=torch.int32, device="cuda"), i32([1, 0, 1500]), 0.1, lse=lse)
    assert (got[1] == 0).all() and (lse[1] == -math.inf).all()
    assert got[::2].isnan().all() and lse[::2].isnan().all()
