"""Parity of the paged cache's operators (vla_cache.h) with their 64-bit oracle, element by element: plans exactly, the
computed outputs within one rounding to their type plus the fp32 error of the sums behind them."""
import math

import numpy as np
import pytest
import torch

from gpu_util import Setup, log
from oracle import cache_oracle as co
from paper_2505_18719_amd import inputs, vla

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24  # unit roundoff of fp32
PAGE = 16
BF, FP = torch.bfloat16, torch.float16


def half_step(ref, dtype):
    """Half a step of dtype at ref: the error of one rounding."""
    f = torch.finfo(dtype)
    return np.maximum(np.abs(ref) * f.eps / 2, f.smallest_normal * f.eps / 2)


def f64(t):
    return t.detach().cpu().double().numpy()


def i32(x):
    return torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()


def rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


# ------------------------------------------------------------------ plan
def run_plan(cached, new, table, free, n_pages, max_rows, head=None, spare_cols=0):
    n, width = table.shape
    wide = np.full((n, width + spare_cols), 123456)
    wide[:, :width] = table
    t = i32(wide)[:, :width] if spare_cols else i32(wide)
    out = vla.kv_plan(i32(cached), i32(new), t, i32(free), n_pages, max_rows, free_head=None if head is None else i32([head]))
    ref, after = co.kv_plan(cached, new, table, free, n_pages, max_rows, head or 0)
    for k, want in ref.items():
        got = out[k].cpu().numpy()
        assert np.array_equal(got, want), (k, np.where(got != want)[0][:8], got[:8], want[:8])
    assert np.array_equal(t.cpu().numpy(), after)
    if spare_cols:
        assert (t.as_strided((n, spare_cols), (width + spare_cols, 1), width).cpu().numpy() == 123456).all()
    return ref


def make_tables(rng, cached, new, extra=2, spare=5):
    held = -(-np.maximum(cached, 0) // PAGE)
    width = int((-(-(np.maximum(cached, 0) + np.maximum(new, 0)) // PAGE)).max(initial=0)) + extra
    need = int((held + -(-np.maximum(new, 0) // PAGE)).sum()) + spare
    pages = rng.permutation(need)
    table, at = np.full((len(cached), width), -1), 0
    for e, h in enumerate(held):
        table[e, :h] = pages[at:at + h]
        at += h
    return table, pages[at:], need


@pytest.mark.parametrize("n,ctx,most,seed", [(255, 30, 9, 11), (256, 30, 9, 12), (257, 30, 9, 13), (1, 0, 1, 0), (1, 37, 1, 1), (1, 15, 500, 2), (7, 40, 60, 3), (64, 400, 1, 4),
                                             (300, 20, 40, 5), (1023, 50, 3, 6), (1024, 50, 3, 7), (1025, 50, 3, 8),
                                             (2500, 33, 9, 9), (3, 0, 70000, 10)])
def test_plan(n, ctx, most, seed):
    rng = np.random.default_rng(seed)
    cached, new = rng.integers(0, ctx + 1, n), rng.integers(0 if n > 1 else 1, most + 1, n)
    table, free, n_pages = make_tables(rng, cached, new)
    run_plan(cached, new, table, free, n_pages, int(new.sum()) + seed, spare_cols=seed % 3)


def test_plan_over_many_workgroups():
    """More rows than one per thread of the largest launch; environments without rows in between."""
    rng = np.random.default_rng(1)
    cached, new = rng.integers(0, 100, 1500), rng.integers(0, 1200, 1500)
    new[rng.integers(0, 1500, 400)] = 0
    table, free, n_pages = make_tables(rng, cached, new)
    run_plan(cached, new, table, free, n_pages, int(new.sum()) + 1000)


@pytest.mark.parametrize("free", [0, 1, 3, 4, 5, 9])
@pytest.mark.parametrize("head", [None, 2])
def test_plan_free_list_runs_out(free, head):
    """Environments are served in order until the pages are gone; those that need none still are."""
    cached, new = np.array([16, 3, 32, 8, 0, 47]), np.array([1, 2, 30, 8, 33, 1])
    table = np.full((6, 6), -1)
    table[:, :3] = np.arange(18).reshape(6, 3)
    pages = list(range(20, 20 + free + (head or 0)))
    out = run_plan(cached, new, table, pages, 64, 80, head)
    need = np.array([1, 0, 2, 0, 3, 0])
    assert out["stats"][2] == ((need > 0) & (need.cumsum() > free)).sum()


@pytest.mark.parametrize("head", [-1, 9, 2 ** 31 - 1])
def test_plan_head_outside_the_list(head):
    out = run_plan(np.array([16, 3]), np.array([1, 2]), np.array([[4, -1], [5, -1]]), list(range(8)), 16, 4, head)
    assert out["lens"].tolist() == [16, 5] and out["stats"].tolist() == [head, 3, 1]


def test_plan_refuses_single_environments():
    """Negative lengths, a sequence past its table row, rows past max_rows: refused, the others served."""
    big = 2 ** 31 - 1
    cached = np.array([5, -1, 5, -7, 60, big, 4, 10, 2])
    new = np.array([3, 2, -4, -1, 5, 3, 2, 50, 1])
    table = np.full((9, 4), -1)
    table[:, 0] = np.arange(9)
    table[4] = [20, 21, 22, 23]
    out = run_plan(cached, new, table, list(range(30, 40)), 64, 20)
    assert out["stats"].tolist() == [0, 20, 7] and out["lens"].tolist() == [8, 0, 5, 0, 60, big, 6, 10, 2]


def test_plan_rows_past_32_bits():
    big = 2 ** 31 - 1
    out = run_plan(np.array([0, 0, 0, 0]), np.array([1, big, big, big]), np.full((4, 3), -1), list(range(9)), 9, 40)
    assert out["row_start"].tolist() == [0, 1, 40, 40, 40] and out["stats"].tolist() == [1, 40, 3]


def test_plan_bad_pages_have_no_slot():
    """Entries and free pages outside the pool are handed on, but their rows have no slot."""
    table = np.array([[99, -1], [-5, -1], [2, -1], [1, -1]])
    run_plan(np.array([3, 3, 15, 15]), np.array([2, 2, 2, 2]), table, [64, 7, -3, 1], 64, 8)
    run_plan(np.array([3, 3, 15, 15]), np.array([2, 2, 2, 2]), table, [2 ** 31 - 1, -2 ** 31], 64, 8)


@pytest.mark.parametrize("n,rows", [(0, 0), (0, 5), (4, 0), (4, 3)])
def test_plan_without_rows(n, rows):
    run_plan(np.full(n, 3), np.zeros(n, int), np.full((n, 2), 1), [], 4, rows)


# ------------------------------------------------------------------ norms, rotation, append
def rope_case(rows, H, K, hd, rot, layout, dtype, norm=(True, True), cache=True, dead=0, far=1000, seed=0, fused=True,
              in_place=False, k_out=False, scale=1.0, eps=1e-6):
    rng = np.random.default_rng(seed)
    if fused:  # parts of one projection's output
        qkv = rand((rows, (H + 2 * K) * hd), dtype, seed, 2.0)
        q, k, v = (t.unflatten(1, (-1, hd)) for t in qkv.split([H * hd, K * hd, K * hd], 1))
    else:
        q, k, v = rand((rows, H, hd), dtype, seed, 2.0), rand((rows, K, hd), dtype, seed + 1), rand((rows, K, hd), dtype, seed + 2)
    gq = (1 + rand((hd,), torch.float32, 5, 0.3)).to(dtype) if norm[0] else None
    gk = (1 + rand((hd,), torch.float32, 6, 0.3)).to(dtype) if norm[1] else None
    pos = rng.integers(0, far + 1, rows)
    freqs = vla.rope_freqs(rot)[0] if rot else None
    n_pages = -(-rows // PAGE) + 3
    slots = rng.permutation(n_pages * PAGE)[:rows] if seed % 2 else np.arange(rows) + seed % 23  # scattered, or runs
    slots[rng.permutation(rows)[:dead]] = rng.choice([-1, -2 ** 31, n_pages * PAGE, 2 ** 31 - 1], dead)
    kp, vp = rand((n_pages, K, PAGE, hd), dtype, 8), rand((n_pages, K, hd, PAGE), dtype, 9)
    old_k, old_v, old_q, old_kk = f64(kp), f64(vp), f64(q), f64(k)
    q_out = q if in_place else torch.full((rows, H, hd), 7.0, dtype=dtype, device="cuda")
    ko = (k if in_place else torch.full((rows, K, hd), 7.0, dtype=dtype, device="cuda")) if k_out or not cache else None
    before_q, before_k = f64(q_out), None if ko is None else f64(ko)
    more = dict(v=v, k_pages=kp, v_pages=vp, row_slot=i32(slots)) if cache else {}
    vla.qk_norm_rope(q, k, i32(pos) if rot else None, freqs, gq, gk, eps, layout, scale, q_out=q_out, k_out=ko, **more)
    torch.cuda.synchronize()
    fr = f64(freqs) if rot else np.zeros(0)
    live = (slots >= 0) & (slots < n_pages * PAGE) if cache else np.full(rows, True)

    def check(got, x, gain, name):
        g = None if gain is None else f64(gain)
        ref = co.norm_turn(x, g, eps, pos, fr, layout, scale)
        y = co.norm_turn(x, g, eps, pos, np.zeros(0), layout)
        mag = np.abs(y)
        if rot:  # a rotated feature has the error of both of its pair
            a, b = co._pairs(rot, layout)
            mag[..., a] = mag[..., b] = abs(scale) * np.hypot(y[..., a], y[..., b])
        # the mean of squares: hd / 16 lanes of 16 sums each, a square root and a division; cos and sin: 4 units, and pi units
        # of the angle that was rounded to fp32 turns; the scale, two products and a sum
        tol = half_step(ref, dtype) * (1 + 2 ** -6) + mag * U32 * (16 + hd / 16 + 24)
        assert np.all(np.abs(got - ref) <= tol), (name, np.max(np.abs(got - ref) / tol))
        return np.max(np.abs(got - ref) / tol)
    gq64, pos = f64(q_out), pos[live]
    worst = check(gq64[live], old_q[live], gq, "q")
    assert np.array_equal(gq64[~live], before_q[~live])
    if ko is not None:
        check(f64(ko)[live], old_kk[live], gk, "k")
        assert np.array_equal(f64(ko)[~live], before_k[~live])
    if cache:
        s = slots[live]
        got_k, got_v = f64(kp), f64(vp)
        check(got_k[s // PAGE, :, s % PAGE], old_kk[live], gk, "k pages")
        assert np.array_equal(got_v[s // PAGE, :, :, s % PAGE], f64(v)[live])
        got_k[s // PAGE, :, s % PAGE] = old_k[s // PAGE, :, s % PAGE]  # and nothing else was written
        got_v[s // PAGE, :, :, s % PAGE] = old_v[s // PAGE, :, :, s % PAGE]
        assert np.array_equal(got_k, old_k) and np.array_equal(got_v, old_v)
    log(f"[rope rows={rows} H={H}/{K} hd={hd} rot={rot} {layout}] worst err/tol {worst}")


@pytest.mark.parametrize("rows,H,K", [(1, 1, 1), (1, 32, 32), (2, 7, 1), (15, 28, 4), (16, 8, 8), (17, 9, 3), (130, 32, 8)])
@pytest.mark.parametrize("hd,rot,layout,dtype", [(128, 128, "half", BF), (64, 64, "interleaved", FP), (256, 256, "half", BF),
                                                 (128, 48, "half", FP), (64, 16, "half", BF), (256, 96, "interleaved", FP),
                                                 (128, 0, "half", BF)])
def test_norm_rope_with_cache(rows, H, K, hd, rot, layout, dtype):
    rope_case(rows, H, K, hd, rot, layout, dtype, dead=min(rows - 1, 3), seed=rows + H + hd // 64)


@pytest.mark.parametrize("norm", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_norm_rope_gains_apart(norm, layout):
    rope_case(37, 6, 2, 128, 64, layout, BF, norm=norm, seed=4)


@pytest.mark.parametrize("cache,k_out,in_place,fused", [(False, True, False, False), (False, True, True, True),
                                                        (True, True, True, True), (True, True, False, False),
                                                        (True, False, True, False)])
def test_norm_rope_outputs(cache, k_out, in_place, fused):
    rope_case(50, 12, 4, 128, 128, "half", BF, cache=cache, k_out=k_out, in_place=in_place, fused=fused, dead=5 if cache else 0,
              seed=3)


@pytest.mark.parametrize("rows", [511, 1025, 2047, 2048, 5000])
@pytest.mark.parametrize("hd,K,dtype", [(64, 4, BF), (128, 8, FP), (256, 1, BF)])
def test_norm_rope_many_rows(rows, hd, K, dtype):
    """On both sides of the split of a row's heads over waves; runs of slots at an odd offset, and scattered ones."""
    for seed in (6, 7):
        rope_case(rows, 2 * K, K, hd, hd, "half", dtype, dead=7, seed=seed)


def test_norm_rope_far_positions_and_scale():
    rope_case(64, 4, 4, 128, 128, "half", BF, far=2 ** 31 - 2, seed=1, scale=1.25)
    rope_case(64, 4, 4, 64, 64, "interleaved", FP, far=4000000, seed=2, scale=-0.5, eps=0.5)


def test_norm_rope_of_zero_and_large_heads():
    """A head of zeros stays zero (eps keeps the norm finite); heads whose squares sum to 1e36 are normed."""
    q = torch.zeros(3, 2, 64, dtype=BF, device="cuda")
    q[1] = 1e17
    q[2, 0, 5] = float("nan")
    g = torch.ones(64, dtype=BF, device="cuda")
    o, _ = vla.qk_norm_rope(q, q.clone(), None, None, g, g)
    assert (o[0] == 0).all() and torch.allclose(o[1].float(), torch.ones(64, device="cuda")) and o[2, 0].isnan().all()
    assert (o[2, 1] == 0).all()  # one head's NaN stays in it


# ------------------------------------------------------------------ backward
def back_case(rows, H, K, hd, rot, layout, dtype, norm=(True, True), fused=True, in_place=False, seed=0, scale=1.0):
    rng = np.random.default_rng(seed)
    width = (H + K) * hd
    x, d = rand((rows, width), dtype, seed, 2.0), rand((rows, width), dtype, seed + 1)
    q, k = (t.unflatten(1, (-1, hd)) for t in x.split([H * hd, K * hd], 1))
    dqo, dko = (t.unflatten(1, (-1, hd)) for t in d.split([H * hd, K * hd], 1))
    if not fused:
        q, k, dqo, dko = (t.contiguous() for t in (q, k, dqo, dko))
    gains = [(1 + rand((hd,), torch.float32, 5 + i, 0.3)).to(dtype) if norm[i] else None for i in range(2)]
    pos = rng.integers(0, 3000, rows)
    freqs = vla.rope_freqs(rot)[0] if rot else None
    fr, eps = f64(freqs) if rot else np.zeros(0), 1e-5
    x64, d64 = (f64(q), f64(k)), (f64(dqo), f64(dko))
    dq, dk = (dqo, dko) if in_place else (None, None)
    first = vla.qk_norm_rope_backward(q if norm[0] else None, k if norm[1] else None, dqo, dko, i32(pos) if rot else None,
                                      freqs, *gains, eps, layout, scale, dq=dq, dk=dk)
    torch.cuda.synchronize()
    worst = 0.0
    for i, name in enumerate(("q", "k")):
        g = None if gains[i] is None else f64(gains[i])
        dx, dg = co.norm_turn_backward(x64[i], g, eps, pos, fr, layout, d64[i], scale)
        mag = np.abs(d64[i])
        if rot:
            a, b = co._pairs(rot, layout)
            mag[..., a] = mag[..., b] = abs(scale) * np.hypot(d64[i][..., a], d64[i][..., b])
        err = mag
        if g is not None:
            r = 1 / np.sqrt((x64[i] ** 2).mean(-1, keepdims=True) + eps)
            h = np.abs(x64[i]) * r
            err = r * (np.abs(g) * mag + 2 * h * (h * np.abs(g) * mag).mean(-1, keepdims=True))
        # as the forward's, and the second mean's sums
        tol = half_step(dx, dtype) * (1 + 2 ** -6) + err * U32 * 2 * (16 + hd / 16 + 24)
        bad = np.abs(f64(first[i]) - dx) / tol
        assert np.all(bad <= 1), (name, bad.max())
        worst = max(worst, bad.max())
        if g is None:
            assert first[2 + i] is None
            continue
        # terms of 64 fp32 errors each, summed in runs of at most rows * heads / 64 + 64
        total = (h * mag).sum((0, 1))
        bad = np.abs(f64(first[2 + i]) - dg) / (total * U32 * (128 + rows * mag.shape[1] / 64))
        assert np.all(bad <= 1), (name + " gain", bad.max())
    if not in_place:
        again = vla.qk_norm_rope_backward(q if norm[0] else None, k if norm[1] else None, dqo, dko,
                                          i32(pos) if rot else None, freqs, *gains, eps, layout, scale)
        assert all(a is None or torch.equal(a, b) for a, b in zip(first, again))  # fixed order of sums
    log(f"[back rows={rows} H={H}/{K} hd={hd} rot={rot} {layout}] worst err/tol {worst:.3f}")


@pytest.mark.parametrize("rows,H,K", [(1, 1, 1), (3, 28, 4), (5, 9, 3), (300, 32, 8), (2500, 5, 1)])
@pytest.mark.parametrize("hd,rot,layout,dtype", [(128, 128, "half", BF), (64, 64, "interleaved", FP), (256, 256, "half", BF),
                                                 (128, 48, "interleaved", BF), (64, 32, "half", FP), (128, 0, "half", BF)])
def test_norm_rope_backward(rows, H, K, hd, rot, layout, dtype):
    back_case(rows, H, K, hd, rot, layout, dtype, seed=rows)


@pytest.mark.parametrize("hd,K,layout", [(128, 8, "half"), (256, 2, "interleaved"), (64, 16, "half")])
def test_norm_rope_backward_of_many_rows(hd, K, layout):
    """Several tiles of rows to a workgroup, and more bytes than the caches are asked to keep."""
    back_case(9001, 3 * K, K, hd, hd, layout, BF, seed=5)


@pytest.mark.parametrize("norm", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("fused,in_place", [(True, True), (False, False)])
def test_norm_rope_backward_gains_apart_and_in_place(norm, fused, in_place):
    back_case(70, 6, 2, 128, 64, "half", BF, norm=norm, fused=fused, in_place=in_place, seed=2, scale=0.75)


def test_norm_rope_backward_without_rows():
    e = torch.empty(0, 4, 64, dtype=BF, device="cuda")
    g = torch.ones(64, dtype=BF, device="cuda")
    p = torch.empty(0, dtype=torch.int32, device="cuda")
    dq, dk, dqg, dkg = vla.qk_norm_rope_backward(e, e, e, e, p, vla.rope_freqs(64)[0], g, g)
    assert dq.shape == e.shape and (dqg == 0).all() and (dkg == 0).all()


def test_norm_rope_backward_against_differences_of_the_forward():
    """The kernel's forward at x +- h against its backward, in half precision with steps that its rounding does not hide."""
    rows, H, hd = 4, 2, 64
    x, d, g = rand((rows, H, hd), FP, 1), rand((rows, H, hd), FP, 2), (1 + rand((hd,), torch.float32, 3, 0.3)).half()
    pos, f = i32([0, 3, 50, 999]), vla.rope_freqs(64)[0]
    dx, dk, dg, _ = vla.qk_norm_rope_backward(x, x, d, d, pos, f, g, g)
    step = rand((rows, H, hd), torch.float32, 4, 0.05)
    up, down = (x.float() + step).half(), (x.float() - step).half()
    fu, fd = (vla.qk_norm_rope(t, t, pos, f, g, g)[0].double() for t in (up, down))
    diff = float(((fu - fd) * d.double()).sum())
    slope = float((dx.double() * (up.double() - down.double())).sum())
    # 512 roundings of outputs of about 1 to half a step 2^-11 on each side, weighted by d; third-order term of the step
    assert abs(diff - slope) <= 6 * 2.0 ** -11 * math.sqrt(2 * rows * H * hd) + 0.02 * abs(slope) + 0.05


# ------------------------------------------------------------------ attention
def make_cache(lens, K, hd, dtype, seed=0, spoil=True, extra_cols=1):
    """Pools, page table and lengths; slots past the lengths hold NaN, table entries past the last page name none."""
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens)
    held = -(-lens // PAGE)
    n_pages = int(held.sum()) + 3
    pages, at = rng.permutation(n_pages), 0
    table = np.full((len(lens), int(held.max(initial=0)) + extra_cols), -7)
    kp, vp = rand((n_pages, K, PAGE, hd), dtype, seed), rand((n_pages, K, hd, PAGE), dtype, seed + 1)
    for e, h in enumerate(held):
        table[e, :h] = pages[at:at + h]
        at += h
        if spoil and lens[e] % PAGE:
            kp[table[e, h - 1], :, lens[e] % PAGE:] = float("nan")
            vp[table[e, h - 1], :, :, lens[e] % PAGE:] = float("inf")
    return kp, vp, table, lens


def attn_tol(ref, mag, smax, hd, dtype):
    # scores: sums of hd products in fp32; weights kept to 16 bits or more for the products with the values
    return half_step(ref, dtype) * (1 + 2 ** -6) + mag * (2.0 ** -16 + 2 * (hd + 32) * U32 * np.maximum(smax, 1.0)[..., None])


def check_attention(got, lse, q, kp, vp, table, lens, scale, envs=None):
    envs = list(range(len(lens))) if envs is None else envs
    hd = q.shape[2]
    ref, rlse, mag, smax = co.paged_attention(f64(q)[envs], f64(kp), f64(vp), table[envs], np.asarray(lens)[envs], scale)
    bad = np.abs(f64(got)[envs] - ref) / attn_tol(ref, mag, smax, hd, got.dtype)
    assert np.all(bad <= 1), (bad.max(), np.argwhere(bad > 1)[:5])
    if lse is not None:
        g = f64(lse)[envs]
        fin = np.isfinite(rlse)
        assert np.array_equal(np.isneginf(g), np.isneginf(rlse))
        assert np.all(np.abs(g[fin] - rlse[fin]) <= (2 * (hd + 32) * U32 * np.maximum(smax[fin], 1) + 4 * U32 * np.abs(rlse[fin])))
    return bad.max()


def attn_case(lens, H, K, hd, dtype, seed=0, qscale=2.0, strided=False, extra_cols=1):
    kp, vp, table, lens = make_cache(lens, K, hd, dtype, seed, extra_cols=extra_cols)
    n, scale = len(lens), hd ** -0.5
    if strided:
        q = rand((n, (H + 2) * hd), dtype, seed + 2, qscale)[:, hd:(H + 1) * hd].unflatten(1, (H, hd))
        wide = torch.full((n, (H + 1) * hd), 5.0, dtype=dtype, device="cuda")
        out = wide[:, :H * hd].unflatten(1, (H, hd))
        t = i32(np.concatenate([table, table], 1))[:, :table.shape[1]]
    else:
        q, out, t = rand((n, H, hd), dtype, seed + 2, qscale), None, i32(table)
    lse = torch.empty(n, H, device="cuda")
    got = vla.paged_attention(q, kp, vp, t, i32(lens), scale, out=out, lse=lse)
    again = vla.paged_attention(q, kp, vp, t, i32(lens), scale)
    torch.cuda.synchronize()
    assert torch.equal(got, again)
    if strided:
        assert (wide[:, H * hd:] == 5).all()
    worst = check_attention(got, lse, q, kp, vp, table, lens, scale)
    log(f"[attn n={n} max={max(lens)} H={H}/{K} hd={hd}] worst err/tol {worst:.3f}")


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 300]


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("H,K", [(1, 1), (7, 7), (8, 2), (28, 4), (16, 1), (17, 1), (40, 1), (64, 1)])
def test_attention_lengths_and_groups(hd, dtype, H, K):
    attn_case(EDGES, H, K, hd, dtype, seed=H + K)


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("H,K", [(1, 1), (7, 7), (8, 2), (28, 4), (17, 1), (40, 1)])
def test_attention_with_room_in_the_table(hd, dtype, H, K):
    """The same lengths in a table with room for more: the keys are split, and nothing of the unused columns is read."""
    attn_case(EDGES, H, K, hd, dtype, seed=H + K, extra_cols=80)


@pytest.mark.parametrize("extra_cols", [1, 80])
@pytest.mark.parametrize("lens,H,K,hd,dtype", [(EDGES * 7, 16, 8, 128, BF), (EDGES * 3, 32, 32, 64, FP), (EDGES * 13, 4, 4, 256, FP),
                                               ([700, 3, 0, 90] * 20, 8, 8, 128, FP), ([1] * 1100, 2, 1, 64, BF)])
def test_attention_of_many_environments(lens, H, K, hd, dtype, extra_cols):
    """From about 1000 key heads in all on, a wave takes one by itself; split, pieces begin and end anywhere in a wave's run."""
    attn_case(lens, H, K, hd, dtype, seed=len(lens), extra_cols=extra_cols)


@pytest.mark.parametrize("n", [1, 2, 3])
@pytest.mark.parametrize("length", [1, 16, 278, 511, 512, 513, 1024, 2047, 4100])
def test_attention_of_few_environments(n, length):
    attn_case([length] * n, 8, 2, 128, BF, seed=n + length)


@pytest.mark.parametrize("lens,H,K,hd,dtype", [([70001, 3], 7, 1, 128, BF), ([33000], 4, 4, 64, FP), ([20011, 0, 9000], 2, 1, 256, BF),
                                               ([5000] + [1] * 200, 4, 1, 128, BF), ([40, 3000, 17] * 30, 8, 8, 64, FP)])
def test_attention_long_and_ragged(lens, H, K, hd, dtype):
    attn_case(lens, H, K, hd, dtype, seed=len(lens), strided=True)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("n", [1, 70000])
def test_attention_of_one_strong_key_among_weak_ones(n, dtype):
    """One key far above n others whose weights, each tiny, add up: they must not be lost to the type of the weights."""
    hd, lens = 64, [n + 1]
    kp, vp, table, lens = make_cache(lens, 1, hd, dtype, 3)
    q = torch.zeros(1, 1, hd, dtype=dtype, device="cuda")
    q[..., 0] = 8.0
    kp[..., 0] = 0.0
    first = table[0, 0]
    kp[first, 0, 0, 0] = 1.75  # score 14 above the others
    vp[first, 0, :, :2] = 1.0
    got = vla.paged_attention(q, kp, vp, i32(table), i32(lens), 1.0)
    check_attention(got, None, q, kp, vp, table, lens, 1.0)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_attention_tail_of_tiny_weights(dtype):
    """200000 keys of weights 2^-29.2 of the strongest key's, whose value is zero: the output is theirs alone."""
    hd, n = 64, 200001
    kp, vp, table, lens = make_cache([n], 1, hd, dtype, 3)
    q = torch.zeros(1, 1, hd, dtype=dtype, device="cuda")
    q[..., 0] = 20.3125
    kp[..., 0] = 0.0
    kp[table[0, 0], 0, 0, 0] = 1.0
    vp[:] = torch.where(torch.isfinite(vp), 1.0, vp)
    vp[table[0, 0], 0, :, 0] = 0.0
    got = f64(vla.paged_attention(q, kp, vp, i32(table), i32(lens), 1.0))
    w = (n - 1) * math.exp(-float(q[0, 0, 0]))  # bf16 holds 20.25
    ref = np.full(got.shape, w / (1 + w))
    # half-precision weights are whole multiples of 2^-39 of the largest (bf16 pairs: 16 bits of each)
    weights = (n - 1) * 2.0 ** -40 if dtype is FP else 2.0 ** -16 * ref
    assert np.all(np.abs(got - ref) <= half_step(ref, dtype) * (1 + 2 ** -6) + weights + 2 * (hd + 32) * U32 * 20.4 * ref)


def test_attention_counts_every_key_once():
    """Equal scores: the mean of the values, whose integers fp32 adds exactly."""
    for n in (1, 5, 16, 1000, 4097):
        kp, vp, table, lens = make_cache([n], 2, 64, FP, 1)
        rng = np.random.default_rng(n)
        vals = rng.integers(-8, 9, (int(vp.shape[0]), 2, 64, PAGE))
        keep = torch.isfinite(vp.float())
        vp = torch.where(keep, torch.from_numpy(vals).half().cuda(), vp)
        q = torch.zeros(1, 2, 64, dtype=FP, device="cuda")
        got = f64(vla.paged_attention(q, kp, vp, i32(table), i32(lens), 1.0))
        for h in range(2):
            _, v = co.cached(f64(kp), f64(vp), table[0], n, h)
            mean = v.mean(0)
            assert np.all(np.abs(got[0, h] - mean) <= half_step(mean, FP) * (1 + 2 ** -6) + 8 * U32 * np.abs(v).mean(0))


def test_attention_of_masked_scores_and_infinities():
    """Keys of -inf scores count nothing, and where nothing else is left the output is zeros, as for length 0; an environment
    that sees a NaN is NaN, and no other is touched."""
    hd = 64
    kp, vp, table, lens = make_cache([40, 40, 40, 40], 1, hd, BF, 2)
    q = rand((4, 1, hd), BF, 4)
    q[..., 0] = 1.0
    kp[..., 0] = 0.0
    kp[table[1, 0], 0, 3, 0] = float("-inf")
    kp[table[2, :3], 0, :, 0] = float("-inf")
    kp[table[3, 1], 0, 5, 7] = float("nan")
    lse = torch.empty(4, 1, device="cuda")
    got = vla.paged_attention(q, kp, vp, i32(table), i32(lens), 1.0, lse=lse)
    check_attention(got, lse, q, kp, vp, table, lens, 1.0, envs=[0, 1])
    assert (got[2] == 0).all() and got[3].isnan().all() and lse[2] == -math.inf and lse[3].isnan()


@pytest.mark.parametrize("long", [False, True])
def test_attention_bad_pages_and_lengths(long):
    """A bad page within the length, a negative length or one past the table: that environment is NaN, the others are right."""
    L = 6000 if long else 90
    lens = [L, L, L - 7, L, 33, L]
    kp, vp, table, lens = make_cache(lens, 2, 128, BF, 5, extra_cols=0)
    q = rand((6, 8, 128), BF, 6)
    table = np.array(table)
    lens = np.array(lens)
    good = table.copy()
    table[1, L // PAGE // 2] = -1
    table[2, 0] = kp.shape[0]
    table[3, (L - 1) // PAGE] = 2 ** 31 - 1
    lens[5] = -1
    lse = torch.empty(6, 8, device="cuda")
    got = vla.paged_attention(q, kp, vp, i32(table), i32(lens), 0.1, lse=lse)
    for e in (1, 2, 3, 5):
        assert got[e].isnan().all() and lse[e].isnan().all()
    check_attention(got, lse, q, kp, vp, good, lens, 0.1, envs=[0, 4])
    lens[5] = table.shape[1] * PAGE + 1
    got = vla.paged_attention(q, kp, vp, i32(table), i32(lens), 0.1)
    assert got[5].isnan().all()
    check_attention(got, None, q, kp, vp, good, lens, 0.1, envs=[0, 4])


def test_attention_without_pages():
    q = rand((3, 4, 64), BF, 1)
    kp = torch.empty(0, 2, PAGE, 64, dtype=BF, device="cuda")
    vp = torch.empty(0, 2, 64, PAGE, dtype=BF, device="cuda")
    got = vla.paged_attention(q, kp, vp, torch.empty(3, 0, dtype=torch.int32, device="cuda"), i32([0, 0, 1]), 1.0)
    assert (got[:2] == 0).all() and got[2].isnan().all()
    got = vla.paged_attention(q, kp, vp, torch.zeros(3, 2, dtype=torch.int32, device="cuda"), i32([0, 0, 1]), 1.0)
    assert (got[:2] == 0).all() and got[2].isnan().all()


def test_attention_shared_pages():
    """Environments that share the pages of a common prefix get what they get with copies of them."""
    kp, vp, table, lens = make_cache([100, 100, 50], 2, 128, BF, 7)
    table = np.array(table)
    table[1, :3], table[2, :3] = table[0, :3], table[0, :3]
    lens = np.array([100, 90, 48])
    q = rand((3, 4, 128), BF, 8)
    got = vla.paged_attention(q, kp, vp, i32(table), i32(lens), 0.1)
    check_attention(got, None, q, kp, vp, table, lens, 0.1)


def test_cache_past_4_gigabytes():
    """Pages whose offsets need more than 32 bits of bytes and of elements: appended to, and read."""
    K, hd, n_pages = 8, 128, 300000  # 9.8 GB a pool, 4.9 G elements
    kp = torch.empty(n_pages, K, PAGE, hd, dtype=BF, device="cuda")
    vp = torch.empty(n_pages, K, hd, PAGE, dtype=BF, device="cuda")
    pages = np.array([299999, 131072, 262144, 131071, 5])
    rows = 70
    q, k, v = rand((rows, K, hd), BF, 1), rand((rows, K, hd), BF, 2), rand((rows, K, hd), BF, 3)
    slots = pages[np.arange(rows) // PAGE] * PAGE + np.arange(rows) % PAGE
    vla.qk_norm_rope(q, k, None, None, v=v, k_pages=kp, v_pages=vp, row_slot=i32(slots))
    got = vla.paged_attention(q[:1], kp, vp, i32([pages]), i32([rows]), 0.2)
    for h in range(K):
        ref, _, mag, smax = co.attention(f64(q)[0, h], f64(k)[:, h], f64(v)[:, h], 0.2)
        assert np.all(np.abs(f64(got)[0, h] - ref) <= attn_tol(ref, mag, np.array(smax), hd, BF))


# ------------------------------------------------------------------ together
class Policy:
    """The attention of a grouped-head decoder layer over a growing cache: random projections of random rows."""

    def __init__(self, envs, H=8, K=2, hd=64, pages=200, width=40, dtype=BF, seed=0):
        self.H, self.K, self.hd, self.dtype = H, K, hd, dtype
        self.kp = torch.full((pages, K, PAGE, hd), float("nan"), dtype=dtype, device="cuda")
        self.vp = torch.full((pages, K, hd, PAGE), float("nan"), dtype=dtype, device="cuda")
        self.table = torch.full((envs, width), -1, dtype=torch.int32, device="cuda")
        self.free = i32(np.random.default_rng(seed).permutation(pages))
        self.lens, self.head = torch.zeros(envs, dtype=torch.int32, device="cuda"), i32([0])
        self.gq, self.gk = ((1 + rand((hd,), torch.float32, s, 0.2)).to(dtype) for s in (1, 2))
        self.freqs, self.scale = vla.rope_freqs(hd, scaling="ramp", factor=4.0, high=32.0, context=256)

    def rows(self, n, seed):
        return rand((n, (self.H + 2 * self.K) * self.hd), self.dtype, seed, 2.0)

    def step(self, qkv, new, plan=None):
        """Plan, append, attend; returns (plan, attention of the rows' environments' last tokens, rotated q)."""
        H, K, hd = self.H, self.K, self.hd
        plan = vla.kv_plan(self.lens, new, self.table, self.free, self.kp.shape[0], qkv.shape[0], free_head=self.head, out=plan)
        q, k, v = (t.unflatten(1, (-1, hd)) for t in qkv.split([H * hd, K * hd, K * hd], 1))
        qo = torch.zeros(qkv.shape[0], H, hd, dtype=self.dtype, device="cuda")
        vla.qk_norm_rope(q, k, plan["row_pos"], self.freqs, self.gq, self.gk, 1e-6, "half", self.scale, v=v, k_pages=self.kp,
                         v_pages=self.vp, row_slot=plan["row_slot"], q_out=qo)
        last = qo[(plan["row_start"][1:] - 1).clamp(min=0).long()]  # the newest row of each environment
        att = vla.paged_attention(last, self.kp, self.vp, self.table, plan["lens"], hd ** -0.5)
        self.lens.copy_(plan["lens"])
        self.head.copy_(plan["stats"][:1])
        return plan, att, last


def reference_step(pol, hist, qkv, new):
    """Appends the rows' keys and values to the environments' histories and attends with the newest row, in 64 bits; keys
    and queries rounded where the cache rounds them."""
    H, K, hd = pol.H, pol.K, pol.hd
    x, f = f64(qkv), f64(pol.freqs)

    def rounded(a):
        return torch.from_numpy(a).to(pol.dtype).double().numpy()
    row, out = 0, np.zeros((len(hist), H, hd))
    tol = np.zeros_like(out)
    for e, w in enumerate(new):
        for _ in range(w):
            p = len(hist[e])
            q = co.norm_turn(x[row, :H * hd].reshape(1, H, hd), f64(pol.gq), 1e-6, [p], f, "half", pol.scale)[0]
            k = co.norm_turn(x[row, H * hd:(H + K) * hd].reshape(1, K, hd), f64(pol.gk), 1e-6, [p], f, "half", pol.scale)[0]
            hist[e].append((rounded(k), x[row, (H + K) * hd:].reshape(K, hd)))
            row += 1
        if w:
            for h in range(H):
                keys = np.array([t[0][h * K // H] for t in hist[e]])
                vals = np.array([t[1][h * K // H] for t in hist[e]])
                o, _, mag, smax = co.attention(rounded(q)[h], keys, vals, hd ** -0.5)
                out[e, h] = o
                # a key or query that the fp32 norm or angle rounds the other way is one step of its type off
                tol[e, h] = attn_tol(o, mag, np.array(smax), hd, pol.dtype) + 4 * torch.finfo(pol.dtype).eps * smax * mag
    return out, tol


def test_a_policy_steps_over_its_cache():
    """A ragged prefill, an idle environment, then decode steps: every environment's attention against its whole history."""
    envs, pol = 5, Policy(5)
    hist = [[] for _ in range(envs)]
    for step, new in enumerate([[20, 1, 47, 16, 0], [1, 1, 1, 0, 33], [1] * 5, [1] * 5, [15, 0, 1, 1, 2], [1] * 5]):
        qkv = pol.rows(sum(new) + 2, step)  # two rows of padding
        plan, att, _ = pol.step(qkv, i32(new))
        ref, tol = reference_step(pol, hist, qkv, new)
        assert plan["lens"].tolist() == [len(h) for h in hist] and int(plan["stats"][2]) == 0
        live = [e for e in range(envs) if new[e]]
        bad = np.abs(f64(att)[live] - ref[live]) / tol[live]
        assert np.all(bad <= 1), (step, bad.max())


def test_a_captured_step_grows_the_cache():
    """One decode step captured into a graph and replayed: lengths, pages and free list advance on the device; every replay
    against the history, with eager work in between."""
    envs, pol = 4, Policy(4, seed=3)
    hist = [[] for _ in range(envs)]
    qkv0 = pol.rows(40, 50)
    pol.step(qkv0, i32([15, 16, 1, 8]))
    reference_step(pol, hist, qkv0, [15, 16, 1, 8])
    static, new = pol.rows(envs, 51), i32([1] * envs)
    keep = [t.clone() for t in (pol.kp, pol.vp, pol.table, pol.lens, pol.head)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        pol.step(static, new)
    torch.cuda.current_stream().wait_stream(s)
    for t, old in zip((pol.kp, pol.vp, pol.table, pol.lens, pol.head), keep):
        t.copy_(old)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        plan, att, _ = pol.step(static, new)
    torch.cuda.synchronize()
    for i in range(6):
        static.copy_(pol.rows(envs, 60 + i))
        g.replay()
        ref, tol = reference_step(pol, hist, static, [1] * envs)
        assert plan["lens"].tolist() == [len(h) for h in hist]
        assert np.all(np.abs(f64(att) - ref) <= tol), i
        torch.randn(1000, device="cuda").sum().item()


def test_a_first_call_may_be_captured():
    """A shape that nothing has run before, in a graph at once (its workgroups take more LDS than a kernel has by default)."""
    kp, vp, table, lens = make_cache([700, 31], 1, 128, FP, 9)
    q, t, n = rand((2, 24, 128), FP, 10), i32(table), i32(lens)
    ws, out = vla.paged_attention_workspace(q, kp, t), torch.empty(2, 24, 128, dtype=FP, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vla.paged_attention(q, kp, vp, t, n, 0.1, out=out, workspace=ws)
    for i in range(3):
        out.zero_()
        n.copy_(i32([lens[0] - 300 * i, lens[1] - i]))
        g.replay()
        check_attention(out, None, q, kp, vp, table, [lens[0] - 300 * i, lens[1] - i], 0.1)


def test_calls_on_another_stream():
    """Operators run on the current stream: work queued there before them is seen, and two streams do not disturb each other."""
    a, b = (make_cache([3000, 700], 2, 128, BF, s) for s in (1, 2))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for i in range(5):
        for s, (kp, vp, table, lens), seed in ((s1, a, 3), (s2, b, 4)):
            with torch.cuda.stream(s):
                q = rand((2, 8, 128), BF, seed)
                got.append((vla.paged_attention(q, kp, vp, i32(table), i32(lens), 0.1), q, kp, vp, table, lens))
    torch.cuda.synchronize()
    for o, q, kp, vp, table, lens in got[-2:]:
        check_attention(o, None, q, kp, vp, table, lens, 0.1)
    assert all(torch.equal(o[0], got[i % 2][0]) for i, o in enumerate(got))


def test_attention_over_a_models_own_cache():
    """The handle's cache has the operators' layout: attention of each environment's last prefix row over the pages that a
    prefill wrote is the attention output of that row in the prefill."""
    S = Setup(inputs.TINY, seed=1)
    cfg, m = S.cfg, S.model
    inp, dev = S.inputs(seed=2)
    B, H, hd = inp.batch, cfg.n_heads, cfg.head_dim
    rows, n_pages = int(inp.prefix_lens.sum()), -(-cfg.max_seq // PAGE) * cfg.batch
    m.debug_layer_limit(1)
    m.debug_stop(2)
    m.prefill(dev["vis"], dev["ids"], inp.prompt_lens)
    q = m.debug_read(1, 0, torch.empty(rows, H, hd, dtype=BF, device="cuda"))
    kp = m.debug_read(2, 0, torch.empty(n_pages, H, PAGE, hd, dtype=BF, device="cuda"))
    vp = m.debug_read(3, 0, torch.empty(n_pages, H, hd, PAGE, dtype=BF, device="cuda"))
    d = cfg.d_model
    u = m.debug_read(4, 0, torch.empty(-(-rows // 16) * (d // 32 + 1) * 512, dtype=BF, device="cuda"))
    m.debug_stop(0)
    m.debug_layer_limit(0)
    u = u.view(-1, d // 32 + 1, 4, 16, 8)[:, :-1].permute(0, 3, 1, 2, 4).reshape(-1, d)  # frag layout back to rows
    last = torch.from_numpy(np.cumsum(inp.prefix_lens) - 1).cuda()
    table = i32(np.arange(n_pages // B)[None] * B + np.arange(B)[:, None])  # page p of environment b is page p B + b
    att = vla.paged_attention(q[last], kp, vp, table, i32(inp.prefix_lens), hd ** -0.5)
    ref, _, mag, smax = co.paged_attention(f64(q[last]), f64(kp), f64(vp), table.cpu().numpy(), inp.prefix_lens, hd ** -0.5)
    tol = attn_tol(ref, mag, smax, hd, BF)
    assert np.all(np.abs(f64(att) - ref) <= tol)
    assert np.all(np.abs(f64(u[last]).reshape(B, H, hd) - f64(att)) <= 2 * tol)


def test_binding_refusals():
    """A small workspace, a host tensor, another type or shape raises and launches nothing."""
    kp, vp, table, lens = make_cache([30], 1, 64, BF, 1)
    q = rand((1, 1, 64), BF, 2)
    with pytest.raises(vla.VlaError) as e:
        vla.paged_attention(q, kp, vp, i32(table), i32(lens), 0.1, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -3
    for bad in (lambda: vla.paged_attention(q, kp, vp, i32(table), i32(lens).cpu(), 0.1),
                lambda: vla.paged_attention(q.half(), kp, vp, i32(table), i32(lens), 0.1),
                lambda: vla.paged_attention(q, kp, vp[:1], i32(table), i32(lens), 0.1),
                lambda: vla.paged_attention(q, kp, vp, i32(table).long(), i32(lens), 0.1),
                lambda: vla.qk_norm_rope(q, q[:, :, ::2], i32([0]), vla.rope_freqs(64)[0]),
                lambda: vla.qk_norm_rope(q, q, i32([0, 1]), vla.rope_freqs(64)[0]),
                lambda: vla.qk_norm_rope(q, q, i32([0]), vla.rope_freqs(64)[0], v_pages=vp),
                lambda: vla.qk_norm_rope_backward(q, q, q, q, i32([0]), vla.rope_freqs(64)[0].float())):
        with pytest.raises(ValueError):
            bad()
