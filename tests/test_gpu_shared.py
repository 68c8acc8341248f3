"""Parity of attention over shared pages (vla_cache.h) with the paged cache's 64-bit oracle: within one rounding to its type, the
rounding of the shared pages' weights, and the fp32 error of the sums."""
import numpy as np
import pytest
import torch

from gpu_util import log
from oracle import cache_oracle as co
from paper_2505_18719_amd import vla
from test_gpu_cache import BF, FP, PAGE, U32, attn_tol, f64, i32, rand

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


class Case:
    """Groups [(shared pages, own tokens of each member)], environments of no group in front and behind; slots past the lengths
    hold NaN, table entries past the last page name none."""

    def __init__(self, groups, K, hd, dtype, seed=0, front=0, behind=0, extra_cols=1):
        rng = np.random.default_rng(seed)
        lone = [(0, [int(n)]) for n in rng.integers(1, 60, front + behind)]
        rows = lone[:front] + list(groups) + lone[front:]
        self.start = np.cumsum([front] + [len(g[1]) for g in groups])
        self.shared = np.array([g[0] for g in groups])
        self.lens = np.array([PAGE * s + n for s, own in rows for n in own])
        own_pages = [-(-n // PAGE) for _, own in rows for n in own]
        width = max([s + -(-n // PAGE) for s, own in rows for n in own]) + extra_cols
        n_pages = sum(s for s, _ in rows) + sum(own_pages) + 3
        pages, at = rng.permutation(n_pages), 0
        self.table = np.full((len(self.lens), width), -7)
        self.kp, self.vp = rand((n_pages, K, PAGE, hd), dtype, seed), rand((n_pages, K, hd, PAGE), dtype, seed + 1)
        e = 0
        for s, own in rows:
            first = pages[at:at + s]
            at += s
            for n in own:
                held = -(-n // PAGE)
                self.table[e, :s] = first
                self.table[e, s:s + held] = pages[at:at + held]
                at += held
                if n % PAGE:
                    self.kp[self.table[e, s + held - 1], :, n % PAGE:] = NAN
                    self.vp[self.table[e, s + held - 1], :, :, n % PAGE:] = INF
                e += 1
        self.n, self.K, self.hd, self.dtype = e, K, hd, dtype

    def run(self, q, scale, lens=None, **more):
        lens = self.lens if lens is None else lens
        return vla.shared_attention(q, self.kp, self.vp, i32(self.table), i32(lens), i32(self.start), i32(self.shared), scale, **more)

    def tol(self, ref, mag, smax):
        """attn_tol, weights once rounded to the type, long sums in fp32."""
        return attn_tol(ref, mag, smax, self.hd, self.dtype) + mag * (torch.finfo(self.dtype).eps / 2 + self.lens.max() * U32)

    def check(self, H, seed=5, scale=None, strided=False):
        scale = self.hd ** -0.5 if scale is None else scale
        hd, n = self.hd, self.n
        q, out = rand((n, H, hd), self.dtype, seed, 2.0), None
        if strided:
            q = rand((n, (H + 2) * hd), self.dtype, seed, 2.0)[:, hd:(H + 1) * hd].unflatten(1, (H, hd))
            wide = torch.full((n, (H + 1) * hd), 5.0, dtype=self.dtype, device="cuda")
            out = wide[:, :H * hd].unflatten(1, (H, hd))
        lse = torch.empty(n, H, device="cuda")
        got = self.run(q, scale, out=out, lse=lse)
        assert torch.equal(got, self.run(q, scale))  # the same bits every run
        if strided:
            assert (wide[:, H * hd:] == 5).all()
        ref, rlse, mag, smax = co.paged_attention(f64(q), f64(self.kp), f64(self.vp), self.table, self.lens, scale)
        bad = np.abs(f64(got) - ref) / self.tol(ref, mag, smax)
        assert np.all(bad <= 1), (bad.max(), np.argwhere(~(bad <= 1))[:5])
        z, fin = f64(lse), np.isfinite(rlse)
        assert np.array_equal(np.isneginf(z), np.isneginf(rlse))
        err = 2 * (hd + 32) * U32 * np.maximum(smax[fin], 1) + 4 * U32 * np.abs(rlse[fin]) + self.lens.max() * U32
        assert np.all(np.abs(z[fin] - rlse[fin]) <= err)
        return bad.max()


GROUPS = [[(1, [1, 16, 17])], [(4, [0, 5]), (5, [40, 0, 3, 100, 64])], [(17, [1] * 9), (0, [20, 3, 4]), (3, [0, 0, 1])],
          [(64, [30, 31]), (7, [200, 1, 2, 33] * 6), (19, [7] * 40)], [(300, list(range(0, 130, 2)))]]


@pytest.mark.parametrize("groups", GROUPS, ids=lambda g: f"{len(g)}groups_{sum(len(x[1]) for x in g)}envs")
@pytest.mark.parametrize("H,K", [(1, 1), (8, 2), (7, 1), (20, 1), (40, 1)])
@pytest.mark.parametrize("hd,dtype", [(64, BF), (128, BF), (256, BF), (128, FP), (64, FP), (256, FP)])
def test_groups(groups, H, K, hd, dtype):
    c = Case(groups, K, hd, dtype, seed=H + hd, front=K, behind=2 if len(groups) % 2 else 0)
    log(f"[shared n={c.n} H={H}/{K} hd={hd}] worst err/tol {c.check(H, strided=H == 8):.3f}")


@pytest.mark.parametrize("groups,H,K,hd,dtype", [([(2000, [5, 9, 70])], 4, 1, 128, BF), ([(12, [3] * 33)] * 30, 16, 8, 64, FP),
                                                 ([(1, [2000, 3])] + [(20, [1, 1])] * 40, 8, 8, 128, BF), ([(9, [1] * 500)], 2, 2, 256, FP),
                                                 ([(5, [8, 8])] * 300, 2, 1, 64, BF), ([(40, [900, 30, 1500])], 8, 4, 128, FP)])
@pytest.mark.parametrize("extra_cols", [1, 60])
def test_many_and_long(groups, H, K, hd, dtype, extra_cols):
    Case(groups, K, hd, dtype, seed=len(groups), extra_cols=extra_cols).check(H)


@pytest.mark.parametrize("scale", [-0.4, 0.0, 2.0])
def test_scales(scale):
    for dtype in (BF, FP):
        Case(GROUPS[1], 2, 64, dtype, seed=3).check(4, scale=scale)


def test_no_groups_and_empty_ones():
    """Without groups, or with one environment in each, the bits are paged_attention's."""
    for groups in ([(0, [3, 70])], [(2, [5]), (7, [1])]):
        c = Case(groups, 2, 64, BF, seed=1)
        q = rand((c.n, 4, 64), BF, 1)
        if len(groups) == 1:
            c.start, c.shared = np.array([0]), np.array([], dtype=int)
        assert torch.equal(c.run(q, 0.1), vla.paged_attention(q, c.kp, c.vp, i32(c.table), i32(c.lens), 0.1))
    c = Case([(4, [5, 9, 1]), (2, [1, 2])], 2, 64, BF, seed=2, front=1, behind=1)
    c.start, c.shared = np.array([1, 1, 4, 4, 6, 6]), np.array([9, 4, -3, 2, 1])
    c.check(8)


def test_lengths_and_pages_that_are_refused():
    """Lengths of zero give zeros; those outside the table, or shorter than what the group shares, NaN, as do pages outside the pool:
    for the whole group if it shares them."""
    c = Case([(4, [5, 9, 1, 7, 3, 8]), (3, [20, 30, 2]), (2, [1, 1])], 2, 128, BF, seed=4)
    lens = c.lens.copy()
    lens[0], lens[1], lens[2], lens[3] = 0, -5, 63, 16 * c.table.shape[1] + 1
    c.table[5, 4] = len(c.kp)       # an own page
    c.table[6:9, 1] = -1            # a page that the group shares
    lens[8] = 0
    q = rand((c.n, 8, 128), BF, 1)
    lse = torch.zeros(c.n, 8, device="cuda")
    got, lse = f64(c.run(q, 0.1, lens=lens, lse=lse)), f64(lse)
    assert (got[[0, 8]] == 0).all() and np.isneginf(lse[[0, 8]]).all()
    assert np.isnan(got[[1, 2, 3, 5, 6, 7]]).all() and np.isnan(lse[[1, 2, 3, 5, 6, 7]]).all()
    ok = [4, 9, 10]
    ref, _, mag, smax = co.paged_attention(f64(q)[ok], f64(c.kp), f64(c.vp), c.table[ok], lens[ok], 0.1)
    assert np.all(np.abs(got[ok] - ref) <= c.tol(ref, mag, smax))
    empty = torch.empty((0, 2, 16, 128), dtype=BF, device="cuda"), torch.empty((0, 2, 128, 16), dtype=BF, device="cuda")
    out = vla.shared_attention(q, *empty, i32(c.table), i32(lens), i32(c.start), i32(c.shared), 0.1)
    assert (f64(out)[[0, 8]] == 0).all() and np.isnan(f64(out)[[1, 4, 10]]).all()


@pytest.mark.parametrize("hd", [64, 128, 256])
def test_not_finite_elements_stay_where_they_belong(hd):
    """In shared pages: the features and key heads of the group only; in own pages: as paged_attention has them."""
    groups = [(6, [5, 40, 1]), (3, [20, 2])]
    for value in (NAN, INF):
        c = Case(groups, 2, hd, BF, seed=7)
        q = rand((c.n, 4, hd), BF, 1)
        clean = f64(c.run(q, 0.1))
        c.vp[c.table[0, 2], 1, 9, 3] = value
        c.vp[c.table[4, 3], 0, 11, 1] = value
        got = f64(c.run(q, 0.1))
        hit = np.zeros(got.shape, bool)
        hit[:3, 2:, 9] = True
        hit[4, :2, 11] = True
        assert not np.isfinite(got[hit]).any() and np.array_equal(got[~hit], clean[~hit])
        assert (got[4, :2, 11] == INF).all() if value == INF else np.isnan(got[4, :2, 11]).all()
    c = Case(groups, 2, hd, FP, seed=8)
    q = rand((c.n, 4, hd), FP, 1).abs()
    c.kp[c.table[0, 0], 0, 5, 0] = -INF  # no weight
    keys = c.kp.clone()
    got = f64(c.run(q, 0.1))
    ref, _, mag, smax = co.paged_attention(f64(q), f64(keys), f64(c.vp), c.table, c.lens, 0.1)
    smax = np.where(np.isfinite(smax), smax, 10.0)
    assert np.all(np.abs(got - ref) <= c.tol(ref, mag, smax))


def test_streams_and_graph():
    """A captured call replayed on new queries and lengths, and the same call on another stream, give an eager call's bits."""
    c = Case([(20, [5, 40, 1, 9]), (33, [20, 2, 2])], 2, 128, BF, seed=7, extra_cols=4)
    q, lens, out = rand((c.n, 8, 128), BF, 1), i32(c.lens), torch.empty((c.n, 8, 128), dtype=BF, device="cuda")
    table, start, shared = i32(c.table), i32(c.start), i32(c.shared)
    ws = vla.shared_attention_workspace(q, c.kp, table, start)
    args = (q, c.kp, c.vp, table, lens, start, shared, 0.08)
    vla.shared_attention(*args, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vla.shared_attention(*args, out=out, workspace=ws)
    for seed in (3, 4, 5):
        q.copy_(rand(q.shape, BF, seed))
        lens.copy_(i32(np.maximum(c.lens - seed, 16 * np.repeat(c.shared, np.diff(c.start)))))
        graph.replay()
        first = out.clone()
        assert torch.equal(first, vla.shared_attention(*args))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            other = vla.shared_attention(*args)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(other, first)


def test_samples_of_one_observation_step_by_step():
    """As sampling continuations runs: one prompt through plan, norms, rotation and prompt attention; its whole pages shared by the
    samples, what is left of it copied to each; then steps of one new token each."""
    H, K, hd, n, prompt, eps = 8, 2, 64, 5, 45, 1e-6
    kp = torch.full((60, K, PAGE, hd), NAN, dtype=BF, device="cuda")
    vp = torch.full((60, K, hd, PAGE), NAN, dtype=BF, device="cuda")
    free, table = i32(np.random.default_rng(0).permutation(60)), i32(np.full((1, 8), -1))
    freqs, _ = vla.rope_freqs(hd)
    gain = torch.ones(hd, dtype=BF, device="cuda")

    def rows(count, seed, plan):
        qkv = rand((count, (H + 2 * K) * hd), BF, seed)
        q, k, v = (t.unflatten(1, (-1, hd)) for t in qkv.split([H * hd, K * hd, K * hd], 1))
        k_out = torch.empty((count, K, hd), dtype=BF, device="cuda")
        q, k = vla.qk_norm_rope(q, k, plan["row_pos"], freqs, gain, gain, eps, v=v, k_pages=kp, v_pages=vp,
                                row_slot=plan["row_slot"], k_out=k_out)
        return q, k, v
    plan = vla.kv_plan(i32([0]), i32([prompt]), table, free, 60, prompt)
    q, k, v = rows(prompt, 1, plan)
    out = vla.prompt_attention(q, k, v, plan["row_start"], 0.125)
    last = vla.paged_attention(q[-1:].contiguous(), kp, vp, table, plan["lens"], 0.125)
    assert np.abs(f64(out[-1]) - f64(last[0])).max() < 0.03  # the same sums; weights rounded once or in pairs
    head = int(plan["stats"][0])
    whole, rest = prompt // PAGE, int(table[0, prompt // PAGE])
    copies = free[head:head + n].long()
    kp[copies], vp[copies] = kp[rest].clone(), vp[rest].clone()
    tables = table.repeat(n, 1)
    tables[:, whole] = copies.int()
    lens, at = i32([prompt] * n), i32([head + n])
    start, shared = i32([0, n]), i32([whole])
    for step in range(6):
        plan = vla.kv_plan(lens, i32([1] * n), tables, free, 60, n, free_head=at)
        lens, at = plan["lens"], plan["stats"][:1].clone()
        q, _, _ = rows(n, 10 + step, plan)
        got = vla.shared_attention(q, kp, vp, tables, lens, start, shared, 0.125)
        ref, _, mag, smax = co.paged_attention(f64(q), f64(kp), f64(vp), tables.cpu().numpy(), lens.cpu().numpy(), 0.125)
        assert np.all(np.abs(f64(got) - ref) <= attn_tol(ref, mag, smax, hd, BF) + mag * 2.0 ** -9)


@pytest.mark.parametrize("H", [1, 3])
def test_most_environments(H):
    """65535 environments, the most that a call takes, in groups of 2 and 3 over 50 pages that all share; some against 64 bits."""
    n, hd, scale = 65535, 64, 0.125
    start = np.concatenate([np.arange(0, 60000, 2), np.arange(60000, n, 3), [n]])
    rng = np.random.default_rng(3)
    shared = rng.integers(1, 4, len(start) - 1)
    group = np.repeat(np.arange(len(shared)), np.diff(start))
    lens = PAGE * shared[group] + rng.integers(0, 17, n)
    table = rng.integers(0, 50, (len(shared), 3))[group]
    table = np.concatenate([table, np.zeros((n, 1), table.dtype)], 1)
    table[np.arange(n), shared[group]] = rng.integers(0, 50, n)
    kp, vp, q = rand((50, 1, PAGE, hd), BF, 1), rand((50, 1, hd, PAGE), BF, 2), rand((n, H, hd), BF, 3, 2.0)
    got = f64(vla.shared_attention(q, kp, vp, i32(table), i32(lens), i32(start), i32(shared), scale))
    some = np.concatenate([np.arange(100), np.arange(59950, 60050), np.arange(n - 100, n)])
    ref, _, mag, smax = co.paged_attention(f64(q)[some], f64(kp), f64(vp), table[some], lens[some], scale)
    tol = attn_tol(ref, mag, smax, hd, BF) + mag * (torch.finfo(BF).eps / 2 + lens.max() * U32)
    assert np.all(np.abs(got[some] - ref) <= tol)
    whole = f64(vla.paged_attention(q, kp, vp, i32(table), i32(lens), scale))
    assert np.isfinite(got).all() and np.abs(got - whole).max() < 0.1  # no row of another environment
