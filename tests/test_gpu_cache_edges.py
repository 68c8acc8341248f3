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


# ------------------------------------------------------------------ infinite and NaN values
# (environments' lengths, heads, key heads, head_dim, columns of the table past the lengths): taken whole by four waves and by
# one, split with a piece in many workgroups, split with many pieces in a wave's run
PATHS = [([90, 33, 1, 500], 8, 2, 128, 1), ([40, 3, 100] * 100, 4, 4, 64, 1), ([3000, 0, 700], 8, 2, 128, 1),
         ([40, 3, 100, 17] * 300, 4, 2, 64, 80), ([900, 70], 6, 1, 256, 1), ([50, 400], 40, 1, 64, 1), ([60, 5000], 40, 1, 128, 1)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lens,H,K,hd,extra_cols", PATHS)
def test_heads_without_a_score_are_zeros_whatever_the_values(lens, H, K, hd, extra_cols, dtype):
    """Every score of the odd key heads is -inf: zeros, with infinities and NaN among the values; the even ones are as ever."""
    kp, vp, table, lens = make_cache(lens, K, hd, dtype, 3, extra_cols=extra_cols)
    q = rand((len(lens), H, hd), dtype, 4)
    q[..., 0] = 1.0
    odd = np.arange(H) * K // H % 2 == 1 if K > 1 else np.full(H, True)
    keys = slice(1, None, 2) if K > 1 else slice(None)
    kp[:, keys, :, 0] = -math.inf
    vp[:, keys, 0::3] = math.inf
    vp[:, keys, 1::3] = math.nan
    lse = torch.empty(len(lens), H, device="cuda")
    got = vla.paged_attention(q, kp, vp, i32(table), i32(lens), hd ** -0.5, lse=lse)
    assert (got[:, odd] == 0).all() and (lse[:, odd] == -math.inf).all()
    if K > 1:
        even = np.arange(K) % 2 == 0
        check_attention(got[:, ~odd], lse[:, ~odd], q[:, ~odd], kp[:, even], vp[:, even], table, lens, hd ** -0.5)


def check_with_infinities(got, lse, q, kp, vp, table, lens, scale):
    """NaN and infinities where the 64-bit sums have them, all else within the tolerance; log-sum-exp as ever."""
    n, H, hd = q.shape
    with np.errstate(invalid="ignore"):
        ref, rlse, mag, smax = co.paged_attention(f64(q), f64(kp), f64(vp), table, lens, scale)
    g, fin = f64(got), np.isfinite(ref)
    assert np.array_equal(np.isnan(g), np.isnan(ref)), np.argwhere(np.isnan(g) != np.isnan(ref))[:5]
    inf = np.isinf(ref)
    assert np.array_equal(g[inf], ref[inf]) and inf.any()
    tol = attn_tol(np.where(fin, ref, 0), np.where(fin, mag, 0), smax, hd, got.dtype)
    assert np.all(np.abs(g - np.where(fin, ref, 0))[fin] <= tol[fin])
    one = np.isfinite(rlse)
    assert np.all(np.abs(f64(lse) - np.where(one, rlse, 0))[one] <= (2 * (hd + 32) * 2.0 ** -24 * np.maximum(smax, 1) +
                                                                       4 * 2.0 ** -24 * np.abs(np.where(one, rlse, 0)))[one])


def spread_infinities(vp, table, lens, seed):
    """In every environment and key head: feature 0 has one infinity, 1 one of the other sign, 2 three of one sign, 3 both
    signs, 4 a NaN beside one, 5 one at the last token; all others are finite."""
    rng = np.random.default_rng(seed)
    put = {math.inf: [], -math.inf: [], math.nan: []}
    for e, n in enumerate(lens):
        for h in range(vp.shape[1] if n > 0 else 0):
            sign = rng.choice([math.inf, -math.inf])
            where = [(0, sign, rng.integers(n)), (1, -sign, rng.integers(n)), (5, sign, n - 1), (4, math.nan, rng.integers(n))]
            where += [(2, sign, t) for t in rng.integers(0, n, 3)]
            if n > 1:
                a, b = rng.choice(n, 2, replace=False)
                where += [(3, sign, a), (3, -sign, b)]
                where += [(4, sign, a)] if where[3][2] != a else []
            for f, x, t in where:
                put[x].append((table[e, t // PAGE], h, f, t % PAGE))
    for x, at in put.items():
        vp[tuple(torch.from_numpy(c) for c in np.array(at).T)] = x


@pytest.mark.parametrize("equal", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lens,H,K,hd,extra_cols", PATHS)
def test_infinite_values_are_infinite_sums(lens, H, K, hd, extra_cols, dtype, equal):
    """With weights that the type holds exactly (equal scores) and others."""
    kp, vp, table, lens = make_cache(lens, K, hd, dtype, 5, extra_cols=extra_cols)
    spread_infinities(vp, table, lens, 6)
    q = rand((len(lens), H, hd), dtype, 7, 0.0 if equal else 2.0)
    lse = torch.empty(len(lens), H, device="cuda")
    got = vla.paged_attention(q, kp, vp, i32(table), i32(lens), hd ** -0.5, lse=lse)
    check_with_infinities(got, lse, q, kp, vp, table, lens, hd ** -0.5)
    again = vla.paged_attention(q, kp, vp, i32(table), i32(lens), hd ** -0.5)
    assert torch.equal(got.nan_to_num(), again.nan_to_num())


@pytest.mark.parametrize("below", [20.0, 60.0, 200.0])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("n,extra_cols", [(90, 1), (2000, 1), (90, 80)])
def test_infinite_values_of_weak_keys(n, extra_cols, first, dtype, below):
    """A weight that no narrow type holds is a weight: infinities at keys far below the strongest, which comes before or after
    them.  (Weights are above 0 in 64 bits up to about 700 below.)"""
    hd = 64
    kp, vp, table, lens = make_cache([n, n], 1, hd, dtype, 8, extra_cols=extra_cols)
    q = torch.zeros(2, 1, hd, dtype=dtype, device="cuda")
    q[..., 0] = below
    kp[..., 0] = 0.0
    strong, weak = (n - 1, 1) if first else (1, n - 1)
    kp[table[0, strong // PAGE], 0, strong % PAGE, 0] = 1.0
    vp[table[0, weak // PAGE], 0, 3, weak % PAGE] = -math.inf
    vp[table[0, 2], 0, 9, 5] = math.inf
    vp[table[1, 3], 0, 9, 5] = math.inf
    lse = torch.empty(2, 1, device="cuda")
    got = vla.paged_attention(q, kp, vp, i32(table), i32(lens), 1.0, lse=lse)
    check_with_infinities(got, lse, q, kp, vp, table, lens, 1.0)


# ------------------------------------------------------------------ the largest calls
def test_norm_rope_of_the_most_rows():
    """2^26 - 4 rows, the most that one call takes: rows of the ends and beyond 2^32 bytes as in a call of their own."""
    rows, hd = 2 ** 26 - 4, 64
    pick = torch.tensor([0, 1, 2, 3, 2 ** 25 - 1, 2 ** 25, 2 ** 25 + 1, 2 ** 26 - 2 ** 13, rows - 5, rows - 2, rows - 1],
                        device="cuda")
    q = torch.zeros(rows, 1, hd, dtype=BF, device="cuda")
    k = torch.zeros(rows, 1, hd, dtype=BF, device="cuda")
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    q[pick], k[pick] = rand((len(pick), 1, hd), BF, 1), rand((len(pick), 1, hd), BF, 2)
    f = vla.rope_freqs(hd)[0]
    want = vla.qk_norm_rope(q[pick], k[pick], pos[pick], f)
    vla.qk_norm_rope(q, k, pos, f, q_out=q, k_out=k)
    assert torch.equal(q[pick], want[0]) and torch.equal(k[pick], want[1])
    q[pick], k[pick] = 0, 0
    assert not q.any() and not k.any()


def test_plan_of_the_most_environments():
    """2^31 - 1 environments, one tile of which ends past that: only the last one has a row, which no page takes."""
    n = 2 ** 31 - 1
    cached, new = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    new[-1] = 1
    out = vla.kv_plan(cached, new, torch.empty(n, 0, dtype=torch.int32, device="cuda"), i32([7]), 8, 3)
    assert out["stats"].tolist() == [0, 1, 1]
    assert out["row_env"].tolist() == [n - 1, -1, -1] and out["row_slot"].tolist() == [-1] * 3 and out["row_pos"].tolist() == [0] * 3
    assert int(out["row_start"][-1]) == 1 and not out["row_start"][:-1].any() and not out["lens"].any()


# ------------------------------------------------------------------ appends
@pytest.mark.parametrize("dtype,K,hd", [(BF, 3, 64), (FP, 2, 128), (BF, 1, 256)])
@pytest.mark.parametrize("rows,runs", [(1, False), (37, True), (129, False), (600, True)])
def test_appends_without_norm_and_rotation_are_copies(rows, runs, dtype, K, hd):
    """Keys and values as they are, infinities and NaN among them, at runs of slots and at scattered ones; rows with slots
    outside the pool are passed over."""
    rng = np.random.default_rng(rows)
    n_pages = rows // PAGE + 4
    slots = np.arange(rows) + 5 if runs else rng.permutation(n_pages * PAGE)[:rows]
    slots[rng.permutation(rows)[:rows // 9]] = rng.choice([-1, -2 ** 31, n_pages * PAGE, 2 ** 31 - 1], rows // 9)
    q, k, v = rand((rows, K, hd), dtype, 1), rand((rows, K, hd), dtype, 2), rand((rows, K, hd), dtype, 3)
    k[0, 0, :3] = v[rows // 2, 0, :3] = torch.tensor([math.inf, -math.inf, math.nan], device="cuda")
    kp, vp = rand((n_pages, K, PAGE, hd), dtype, 4), rand((n_pages, K, hd, PAGE), dtype, 5)
    want = co.append(f64(kp), f64(vp), slots, f64(k), f64(v))
    vla.qk_norm_rope(q, k, None, None, v=v, k_pages=kp, v_pages=vp, row_slot=i32(slots))
    assert np.array_equal(f64(kp), want[0], equal_nan=True) and np.array_equal(f64(vp), want[1], equal_nan=True)
