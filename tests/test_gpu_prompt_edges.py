"""Edges of attention over whole prompts and its gradient: rows all of whose scores are -inf, a scale of 0."""
import numpy as np
import pytest
import torch

from oracle import prompt_oracle as po
from paper_2505_18719_amd import vla
from test_gpu_cache import BF, FP, U32, f64, half_step
from test_gpu_prompt import INF, NAN, Case, bits

pytestmark = pytest.mark.gpu

KINDS = [(64, BF, 4, 2), (128, BF, 4, 1), (128, FP, 4, 2), (256, BF, 2, 2), (256, FP, 4, 2), (64, FP, 16, 8)]


def against(ref, c, sel=None, sel_kv=None):
    """The gradients of c against the oracle's of ref's inputs."""
    ref.out, ref.dq, ref.dk, ref.dv = c.out, c.dq, c.dk, c.dv
    return ref.check_backward(sel, sel_kv)


@pytest.mark.parametrize("hd,dtype,H,K", KINDS)
@pytest.mark.parametrize("dout", [None, INF, NAN])
def test_queries_of_minus_infinity_give_no_gradient(hd, dtype, H, K, dout):
    """A query with an element of -inf where all keys are above 0 has no weight: its dq is zeros, and dk and dv have nothing of
    it, whatever its own elements and its dout are; wherever it lies to the keys' tiles, and alone or among others."""
    for lens, rows in (([200, 70], [0]), ([200, 70], [40, 199]), ([33, 300, 5], [32, 64, 65, 127, 128, 299]), ([130], [129]),
                       ([64, 1, 1], [63, 64]), ([400], range(0, 400, 3))):
        a, b = (Case(lens, H, K, hd, dtype, seed=len(rows)) for _ in range(2))
        for c in (a, b):
            c.k[:, :, 3] = c.k[:, :, 3].abs() + 0.1
        at = [int(a.start[0]) + r for r in rows]
        a.q[at, :, 3] = -INF
        b.q[at] = 0
        b.dout[at] = 0
        if dout is not None:
            a.dout[at, :, 7] = dout
        a.run()
        out, lse = f64(a.out), f64(a.lse)
        assert (out[at] == 0).all() and np.isneginf(lse[at]).all()
        first = [bits(t) for t in a.back()]
        assert (f64(a.dq)[at] == 0).all()
        against(b, a)
        assert all(torch.equal(x, bits(y)) for x, y in zip(first, a.back()))


@pytest.mark.parametrize("hd,dtype", [(64, BF), (128, FP), (128, BF), (256, BF)])
@pytest.mark.parametrize("n,most", [(70, 140), (600, 5)])
def test_queries_of_minus_infinity_among_many_sequences(n, most, hd, dtype):
    """The same where the keys' workgroups fill the GPU, and where the sequences are more than are listed."""
    rng = np.random.default_rng(n)
    lens = rng.integers(1, most + 1, n)
    a, b = (Case(lens, 8, 4, hd, dtype, seed=n) for _ in range(2))
    for c in (a, b):
        c.k[:, :, 3] = c.k[:, :, 3].abs() + 0.1
    at = rng.choice(np.arange(a.rows)[a.inside], sum(lens) // 5, replace=False)
    a.q[at, ::2, 3] = -INF
    a.dout[at, ::2, 7] = NAN
    b.q[at, ::2] = 0
    b.dout[at, ::2] = 0
    a.run()
    assert (f64(a.out)[at][:, ::2] == 0).all() and np.isneginf(f64(a.lse)[at][:, ::2]).all()
    a.back()
    assert (f64(a.dq)[at][:, ::2] == 0).all()
    against(b, a)


@pytest.mark.parametrize("hd,dtype,H,K", KINDS)
@pytest.mark.parametrize("dout", [None, NAN])
def test_keys_of_minus_infinity_at_the_start(hd, dtype, H, K, dout):
    """Rows that see only keys of -inf: their gradients are zeros in every element, and dk and dv of all keys are those of the
    sequence without them."""
    lens, n = [150, 40], 3
    c = Case(lens, H, K, hd, dtype, seed=9)
    c.q[:, :, 0] = c.q[:, :, 0].abs() + 0.1
    s = int(c.start[0])
    c.k[s:s + n, :, 0] = -INF
    if dout is not None:
        c.dout[s:s + n, :, 5] = dout
        c.v[s:s + n, :, 5] = INF
    ref = Case(lens, H, K, hd, dtype, seed=9)
    for x, y in ((ref.q, c.q), (ref.k, c.k), (ref.v, c.v), (ref.dout, c.dout)):
        x.copy_(y)
    ref.start = ref.start.copy()
    ref.start[0] += n
    c.run()
    c.back()
    assert (f64(c.dq)[s:s + n] == 0).all()
    rows = np.arange(c.rows)
    behind = c.inside & (rows >= c.start[1])  # the other sequence
    kv = behind if dout is not None else c.inside & ((rows < s) | (rows >= s + n))  # an infinite value reaches the rows behind it
    if dout is None:
        assert (f64(c.dk)[s:s + n] == 0).all() and (f64(c.dv)[s:s + n] == 0).all()
    against(ref, c, behind, kv)  # dq of the rows behind the keys: 0 times -inf in one element


@pytest.mark.parametrize("dtype", [BF, FP])
def test_rows_without_weight_beside_bad_elements(dtype):
    """A row without weight, and a NaN that reaches what its formulas say: the two do not meet in other heads and keys."""
    c, clean = Case([300], 4, 2, 128, dtype, seed=3), Case([300], 4, 2, 128, dtype, seed=3)
    s = int(c.start[0])
    for x in (c, clean):
        x.k[:, :, 3] = x.k[:, :, 3].abs() + 0.1
    c.q[s + 250, 3, 3] = -INF
    c.dout[s + 100, 0, 9] = NAN
    clean.q[s + 250, 3] = 0
    clean.dout[s + 250, 3] = 0
    c.run()
    c.back()
    clean.out, clean.lse = c.out, c.lse
    dk, dv = f64(c.dk), f64(c.dv)
    assert np.isnan(dk[s:s + 101, 0]).all() and np.isnan(dv[s:s + 101, 0, 9]).all()
    assert np.isfinite(dk[s + 101:-2, 0]).all() and np.isfinite(dk[s:-2, 1]).all() and np.isfinite(dv[s + 101:-2]).all()
    clean.dq, clean.dk, clean.dv = c.dq, c.dk, c.dv
    g, _ = po.backward(f64(clean.q), f64(clean.k), f64(clean.v), f64(clean.dout), clean.start, clean.scale)
    for got, want in ((dk[s:-2, 1], g[1][s:-2, 1]), (dv[s:-2, 1], g[2][s:-2, 1]), (dk[s + 101:-2, 0], g[1][s + 101:-2, 0])):
        assert np.linalg.norm(got - want) <= 4 * torch.finfo(dtype).eps / 2 * np.linalg.norm(want)
    assert (f64(c.dq)[s + 250, 3] == 0).all()


@pytest.mark.parametrize("hd,dtype,H,K", [(64, BF, 4, 2), (128, FP, 4, 2), (256, BF, 2, 2)])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("what", ["q", "k"])
def test_scale_of_0_times_infinite_elements(what, value, hd, dtype, H, K):
    """0 times an infinite or NaN element is NaN: a query's reaches its row, a key's the rows that see it, and their gradients;
    all else is what it is without them."""
    c, clean = (Case([50, 120], H, K, hd, dtype, seed=4, scale=0.0) for _ in range(2))
    r, head = int(c.start[1]) + 70, 1
    getattr(c, what)[r, head, 11] = value
    for x in (c, clean):
        x.run()
        x.back()
    rows, heads = np.arange(c.rows), np.arange(H)
    hit = (rows[:, None] == r) & (heads == head) if what == "q" else (rows[:, None] >= r) & (heads // (H // K) == head)
    hit &= c.inside[:, None]
    group = np.arange(K) == (head * K // H if what == "q" else head)
    hit_kv = c.inside[:, None] & (rows[:, None] >= c.start[1]) & group  # keys that a row that is hit sees
    if what == "q":
        hit_kv &= rows[:, None] <= r
    for name, where in (("out", hit), ("lse", hit), ("dq", hit), ("dk", hit_kv), ("dv", hit_kv)):
        got, want = f64(getattr(c, name)), f64(getattr(clean, name))
        assert np.isnan(got[where]).all(), name
        bound = 0.0
        if name == "dv":
            # All weights of row i of a sequence are 1 / (i + 1).  A wave's keys beside one that is reached are summed with them in
            # fp32, else rounded to the type (half a step of each term), and both results are rounded once: half a step each.
            mag = np.zeros(want.shape)
            for a, b in zip(c.start, c.start[1:]):
                terms = np.abs(f64(c.dout)[a:b]) / np.arange(1, b - a + 1)[:, None, None]
                mag[a:b] = terms[::-1].cumsum(0)[::-1].reshape(b - a, K, H // K, hd).sum(2)
            bound = 2 * half_step(want, dtype) * (1 + 2 ** -6) + mag * (torch.finfo(dtype).eps / 2 + 2 * 120 * H * U32)
        assert (np.abs(got - want) <= bound)[~where & c.inside[:, None]].all(), name
