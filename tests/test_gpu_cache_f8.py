"""Parity of the cache in 8-bit numbers (vla_cache.h) with its 64-bit oracle: what is stored byte by byte, what is read back bit by
bit, and attention over it within one rounding to its type plus the fp32 error of the sums behind it."""
import numpy as np
import pytest
import torch

from gpu_util import log
from oracle import cache_f8_oracle as c8
from oracle import cache_oracle as co
from paper_2505_18719_amd import vla
from test_gpu_cache import BF, EDGES, FP, PAGE, U32, attn_tol, f64, i32, rand

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def pool(n_pages, K, hd, seed=0):
    """Bytes of all kinds (no NaN) and scales of different sizes, on the device."""
    rng = np.random.default_rng(seed)
    kb, vb = (rng.integers(0, 127, s).astype(np.uint8) | (rng.integers(0, 2, s).astype(np.uint8) << 7)
              for s in ((n_pages, K, PAGE, hd), (n_pages, K, hd, PAGE)))
    ks, vs = (np.exp(rng.normal(size=(n_pages, K, PAGE)) * 0.3 - 5.5).astype(np.float32) for _ in range(2))
    return kb, vb, ks, vs


def to_gpu(p):
    kb, vb, ks, vs = (torch.from_numpy(x).cuda() for x in p)
    return kb.view(F8), vb.view(F8), ks, vs


def same_pool(got, want):
    for g, w in zip(got, want):
        g = (g.view(torch.uint8) if g.dtype is F8 else g.view(torch.int32)).cpu().numpy()
        w = w if w.dtype == np.uint8 else w.view(np.int32)
        nan = (w & 0x7f) == 0x7f if w.dtype == np.uint8 else np.isnan(w.view(np.float32))
        assert np.array_equal(g[~nan], w[~nan]), np.argwhere((g != w) & ~nan)[:4]
        if w.dtype == np.uint8:
            assert ((g[nan] & 0x7f) == 0x7f).all()
        else:
            assert np.isnan(g.view(np.float32)[nan]).all()


def store_case(k, v, slots, n_pages, strided=False):
    rows, K, hd = k.shape
    if strided:
        wide = torch.cat([k.reshape(rows, -1), v.reshape(rows, -1), k.reshape(rows, -1)[:, :8]], 1)
        k, v = (t.unflatten(1, (K, hd)) for t in (wide[:, :K * hd], wide[:, K * hd:2 * K * hd]))
    before = pool(n_pages, K, hd, rows)
    p = to_gpu(before)
    vla.kv_append_f8(k, v, i32(slots), *p)
    after = c8.append(*before, slots, f64(k), f64(v))
    same_pool(p, after)
    ko, vo = (torch.full((rows, K * hd + 8), 7.0, dtype=k.dtype, device="cuda") for _ in range(2))
    kr, vr = vla.kv_read_f8(i32(slots), *p, k_out=ko[:, :K * hd].unflatten(1, (K, hd)), v_out=vo[:, :K * hd].unflatten(1, (K, hd)))
    live = [r for r, s in enumerate(slots) if 0 <= s < PAGE * n_pages]
    s = np.asarray(slots)[live]
    for got, byte, scale in ((kr, after[0][s // PAGE, :, s % PAGE], after[2]), (vr, after[1][s // PAGE, :, :, s % PAGE], after[3])):
        want = c8.NUMBERS[byte].astype(np.float32) * scale[s // PAGE, :, s % PAGE][..., None]
        with np.errstate(over="ignore"):
            want = torch.from_numpy(want).to(k.dtype)
        assert torch.equal(got[live].cpu().nan_to_num(9.0, 99999.0 if k.dtype is BF else 65504.0), want.nan_to_num(9.0, 99999.0 if k.dtype is BF else 65504.0))
        dead = [r for r in range(rows) if r not in set(live)]
        assert (got[dead] == 7).all()
    assert (ko[:, K * hd:] == 7).all() and (vo[:, K * hd:] == 7).all()


@pytest.mark.parametrize("hd,dtype", [(64, BF), (128, BF), (256, BF), (64, FP), (128, FP), (256, FP)])
@pytest.mark.parametrize("K", [1, 3, 8])
def test_store_and_read(hd, dtype, K):
    """Rows anywhere, in runs from any slot on, and outside the pool, of every size the type holds."""
    rng = np.random.default_rng(hd + K)
    for rows in (1, 2, 17, 100, 333, 2100):  # the last in workgroups of 64 rows, with 8 heads
        n_pages = rows // PAGE + 9
        order = rng.permutation(n_pages * PAGE)[:rows]
        start = int(rng.integers(0, 40))
        runs = np.concatenate([np.arange(start, start + rows)])
        pages = (rng.permutation(n_pages)[:, None] * PAGE + np.arange(PAGE)).reshape(-1)[5:5 + rows]
        for slots in (order, runs, pages):
            slots = np.array(slots)
            if rows > 2:
                slots[rng.integers(0, rows, rows // 9 + 1)] = -1
                slots[rng.integers(0, rows)] = n_pages * PAGE
            size = torch.from_numpy(np.exp(rng.normal(size=(rows, K, 1)) * 3)).cuda()
            k, v = ((rand((rows, K, hd), torch.float32, s).double() * size).to(dtype) for s in (rows, rows + 1))
            store_case(k, v, slots, n_pages, strided=rows % 2 == 1)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_store_sizes_ties_and_not_finite(dtype):
    """Zeros, the least and largest numbers of the type, quotients half way between two 8-bit numbers, infinities and NaN."""
    hd, f = 64, torch.finfo(dtype)
    x = torch.zeros(12, 2, hd, dtype=dtype)
    x[1] = f.tiny
    x[2, :, 0], x[2, :, 1:] = f.max, f.tiny
    x[3] = f.max
    x[4, 0, 5], x[4, 1, 7] = float("inf"), float("nan")
    x[5, :, :] = 1.0
    x[5, 1, 63] = float("-inf")
    for r, top in ((6, 7.0), (7, 1.75), (8, 448.0), (9, 0.875)):  # eighths of powers of two and what lies between
        x[r] = torch.tensor([top / 448 * (16 + i % 16) * 2.0 ** (i // 16) / 16 for i in range(hd)]).to(dtype)
        x[r, :, 0] = -top
    x[10] = f.tiny * f.eps if dtype is FP else 2.0 ** -133  # subnormal
    x[11, :, ::2] = -0.0
    x[11, :, 3] = 2.0 ** -14
    store_case(x.cuda(), x.flip(0).contiguous().cuda(), list(range(20, 32)), 4)


def test_store_and_read_nothing():
    p = to_gpu(pool(3, 2, 64))
    e = torch.empty(0, 2, 64, dtype=BF, device="cuda")
    vla.kv_append_f8(e, e, i32([]), *p)
    assert vla.kv_read_f8(i32([]), *p)[0].shape == (0, 2, 64)
    k, v = vla.kv_read_f8(i32([-1, 48]), *p, dtype=FP)
    assert k.dtype is FP and (k == 0).all() and (v == 0).all()


def make_cache(lens, K, hd, seed=0, extra_cols=1):
    """Pools, page table and lengths; slots past the lengths hold NaN, with scales NaN or infinite."""
    rng = np.random.default_rng(seed)
    held = -(-np.asarray(lens) // PAGE)
    n_pages = int(held.sum()) + 3
    pages, at = rng.permutation(n_pages), 0
    table = np.full((len(lens), int(held.max(initial=0)) + extra_cols), -7)
    p = pool(n_pages, K, hd, seed)
    for e, h in enumerate(held):
        table[e, :h] = pages[at:at + h]
        at += h
        if lens[e] % PAGE:
            last, n = table[e, h - 1], lens[e] % PAGE
            p[0][last, :, n:], p[1][last, :, :, n:] = 0x7f, 0xff
            p[2][last, :, n:], p[3][last, :, n:] = np.nan, np.inf
    return p, table


def attn_case(lens, H, K, hd, dtype, seed=0, extra_cols=1, strided=False):
    p, table = make_cache(lens, K, hd, seed, extra_cols)
    n, scale = len(lens), hd ** -0.5
    q, out, t = rand((n, H, hd), dtype, seed + 2, 2.0), None, i32(table)
    if strided:
        q = rand((n, (H + 2) * hd), dtype, seed + 2, 2.0)[:, hd:(H + 1) * hd].unflatten(1, (H, hd))
        wide = torch.full((n, (H + 1) * hd), 5.0, dtype=dtype, device="cuda")
        out = wide[:, :H * hd].unflatten(1, (H, hd))
        t = i32(np.concatenate([table, table], 1))[:, :table.shape[1]]
    lse = torch.empty(n, H, device="cuda")
    g = to_gpu(p)
    got = vla.paged_attention_f8(q, *g, t, i32(lens), scale, out=out, lse=lse)
    assert torch.equal(got, vla.paged_attention_f8(q, *g, t, i32(lens), scale))
    if strided:
        assert (wide[:, H * hd:] == 5).all()
    with np.errstate(invalid="ignore"):
        kv = c8.values(*p)
    ref, rlse, mag, smax = co.paged_attention(f64(q), *kv, table, lens, scale)
    bad = np.abs(f64(got) - ref) / attn_tol(ref, mag, smax, hd, dtype)
    assert np.all(bad <= 1), (bad.max(), np.argwhere(bad > 1)[:5])
    fin = np.isfinite(rlse)
    z = f64(lse)
    assert np.array_equal(np.isneginf(z), np.isneginf(rlse))
    assert np.all(np.abs(z[fin] - rlse[fin]) <= 2 * (hd + 32) * U32 * np.maximum(smax[fin], 1) + 4 * U32 * np.abs(rlse[fin]))
    log(f"[attn f8 n={n} max={max(lens)} H={H}/{K} hd={hd}] worst err/tol {bad.max():.3f}")


@pytest.mark.parametrize("extra_cols", [1, 90])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("H,K", [(1, 1), (7, 7), (28, 4), (17, 1), (40, 1)])
def test_attention_lengths_and_groups(hd, dtype, H, K, extra_cols):
    attn_case(EDGES, H, K, hd, dtype, seed=H + K, extra_cols=extra_cols)


@pytest.mark.parametrize("lens,H,K,hd,dtype", [(EDGES * 7, 16, 8, 128, BF), ([700, 3, 0, 90] * 40, 8, 8, 64, FP), ([70001, 3], 7, 1, 128, BF),
                                               ([33000], 4, 4, 64, FP), ([20011, 0, 9000], 2, 1, 256, BF), ([278], 32, 32, 128, BF),
                                               ([5000] + [1] * 200, 4, 1, 128, FP), ([40, 2900, 17] * 30, 8, 8, 64, BF), ([1040] * 3, 8, 2, 256, FP)])
def test_attention_many_and_long(lens, H, K, hd, dtype):
    attn_case(lens, H, K, hd, dtype, seed=len(lens), strided=True)


def test_attention_of_scales_of_any_size():
    """Keys and values far from 1, in half precision: scales that its range does not hold."""
    for ks, vs in ((1e-6, 1e-9), (3.0, 120.0), (1e-3, 30.0)):
        p, table = make_cache([77, 300, 5], 2, 128, 5)
        p[2][:] *= ks / 0.004
        p[3][:] *= vs / 0.004
        q = rand((3, 8, 128), FP, 1, 0.004 / ks if ks > 1 else 2.0)
        got = vla.paged_attention_f8(q, *to_gpu(p), i32(table), i32([77, 300, 5]), 0.08)
        with np.errstate(invalid="ignore"):
            ref, _, mag, smax = co.paged_attention(f64(q), *c8.values(*p), table, [77, 300, 5], 0.08)
        assert np.all(np.abs(f64(got) - ref) <= attn_tol(ref, mag, smax, 128, FP))


@pytest.mark.parametrize("hd", [64, 128, 256])
def test_attention_refuses_lengths_pages_and_nan(hd):
    """As over 16-bit pages: NaN for a length outside the table or a page outside the pool; NaN elements reach their own heads and
    features only."""
    lens = [40, 70, 33, -1, 200, 33, 33]
    p, table = make_cache([40, 70, 33, 0, 0, 33, 33], 2, hd, 3)
    n_pages = len(p[0])
    table[1, 4], table[2, 0] = n_pages, -1
    p[2][table[5, 1], 1, 3] = np.nan       # a key of head 1
    p[1][table[6, 0], 0, 9, 7] = 0x7f      # feature 9 of a value of head 0
    q = rand((7, 4, hd), BF, 1)
    got = f64(vla.paged_attention_f8(q, *to_gpu(p), i32(table), i32(lens), 0.1))
    assert np.isnan(got[[1, 2, 3, 4]]).all() and np.isfinite(got[0]).all()
    assert np.isfinite(got[5, :2]).all() and np.isnan(got[5, 2:]).all()
    nan = np.isnan(got[6])
    assert nan[:2, 9].all() and nan.sum() == 2


def test_streams_and_graph():
    """Appending and attending captured together and replayed on new tokens, beside eager work on another stream."""
    n, H, K, hd = 5, 8, 2, 128
    lens = [40, 100, 1, 16, 700]
    p, table = make_cache(lens, K, hd, 1, extra_cols=3)
    for x, clean in zip(p, pool(len(p[0]), K, hd, 1)):
        x[:] = clean
    g, t = to_gpu(p), i32(table)
    q, k, v = rand((n, H, hd), BF, 1), rand((n, K, hd), BF, 2), rand((n, K, hd), BF, 3)
    slot = i32([table[e, (lens[e] - 1) // PAGE] * PAGE + (lens[e] - 1) % PAGE for e in range(n)])
    out, ws, lens = torch.empty_like(q), vla.paged_attention_workspace(q, g[0], t), i32(lens)

    def step(to):
        vla.kv_append_f8(k, v, slot, *g)
        vla.paged_attention_f8(q, *g, t, lens, 0.09, out=to, workspace=ws)
    step(out)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(out)
    for seed in (10, 20, 30):
        for i, x in enumerate((q, k, v)):
            x.copy_(rand(x.shape, BF, seed + i))
        graph.replay()
        first = out.clone()
        eager = torch.empty_like(q)
        step(eager)
        assert torch.equal(first, eager)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            other = vla.paged_attention_f8(q, *g, t, lens, 0.09)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(other, eager)


def test_policy_steps_over_an_8_bit_cache():
    """Plans, norms and rotation, appends and attention over several steps, as a decoder layer serves: against the oracle of the
    cache that was stored, and the stored cache against the keys and values that went in."""
    n, H, K, hd, pages, width = 4, 8, 2, 64, 120, 30
    kp = torch.zeros((pages, K, PAGE, hd), dtype=torch.uint8, device="cuda").view(F8)
    vp = torch.zeros((pages, K, hd, PAGE), dtype=torch.uint8, device="cuda").view(F8)
    ks, vs = torch.zeros((pages, K, PAGE), device="cuda"), torch.zeros((pages, K, PAGE), device="cuda")
    table, free, head = i32(np.full((n, width), -1)), i32(np.random.default_rng(1).permutation(pages)), i32([0])
    lens = i32([0] * n)
    freqs, _ = vla.rope_freqs(hd)
    gain = torch.ones(hd, dtype=BF, device="cuda")
    for step, new in enumerate(([37, 0, 80, 5], [1, 20, 1, 1], [1, 1, 1, 1], [1, 1, 1, 1])):
        rows = sum(new)
        plan = vla.kv_plan(lens, i32(new), table, free, pages, rows, free_head=head)
        qkv = rand((rows, (H + 2 * K) * hd), BF, step)
        q, k, v = (t.unflatten(1, (-1, hd)) for t in qkv.split([H * hd, K * hd, K * hd], 1))
        qr, kr = vla.qk_norm_rope(q, k, plan["row_pos"], freqs, gain, gain)
        vla.kv_append_f8(kr, v, plan["row_slot"], kp, vp, ks, vs)
        back_k, back_v = vla.kv_read_f8(plan["row_slot"], kp, vp, ks, vs)
        for got, want in ((back_k, kr), (back_v, v)):
            w = f64(want)
            unit = np.abs(w).max(-1, keepdims=True) / 448
            assert np.all(np.abs(f64(got) - w) <= np.maximum(np.abs(w) * 2.0 ** -4, unit * 2.0 ** -10) + np.abs(w) * 1.1 * 2.0 ** -9)
        lens, head = plan["lens"], plan["stats"][:1].clone()
        last = (plan["row_start"][1:] - 1).clamp(min=0).long()
        qe = qr[last].contiguous()
        got = vla.paged_attention_f8(qe, kp, vp, ks, vs, table, lens, hd ** -0.5)
        pools = c8.values(*(x.view(torch.uint8).cpu().numpy() for x in (kp, vp)), ks.cpu().numpy(), vs.cpu().numpy())
        ref, _, mag, smax = co.paged_attention(f64(qe), *pools, table.cpu().numpy(), lens.cpu().numpy(), hd ** -0.5)
        assert np.all(np.abs(f64(got) - ref) <= attn_tol(ref, mag, smax, hd, BF))
