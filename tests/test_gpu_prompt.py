"""Parity of attention over whole prompts and its gradient (vla_prompt.h) with their 64-bit oracle, element by element:
within one rounding to their type, the rounding of the weights to that type, and the fp32 error of the sums."""
import numpy as np
import pytest
import torch

from gpu_util import log
from oracle import cache_oracle as co
from oracle import prompt_oracle as po
from paper_2505_18719_amd import vla
from test_gpu_cache import BF, FP, U32, f64, half_step, i32, rand

pytestmark = pytest.mark.gpu


def bits(t):
    return t.contiguous().view(torch.int16)


class Case:
    """Packed sequences of the given lengths, `gap` rows in front, behind and NaN there; q, k and v parts of one projection if
    `joint`."""

    def __init__(self, lens, H, K, hd, dtype, seed=0, scale=None, qscale=2.0, gap=2, joint=True):
        self.start = np.concatenate([[0], np.cumsum(lens)]) + gap
        self.rows, self.H, self.K, self.hd, self.dtype = int(self.start[-1]) + gap, H, K, hd, dtype
        self.scale = hd ** -0.5 if scale is None else scale
        width = (H + 2 * K) * hd
        x = rand((self.rows, width + 16), dtype, seed)[:, 8:8 + width]
        self.q, self.k, self.v = (t.unflatten(1, (-1, hd)) for t in x.split([H * hd, K * hd, K * hd], 1))
        if not joint:
            self.q, self.k, self.v = (t.contiguous() for t in (self.q, self.k, self.v))
        self.q.mul_(qscale)
        self.dout = rand((self.rows, H * hd), dtype, seed + 1, 0.1).unflatten(1, (H, hd))
        inside = np.zeros(self.rows, bool)
        inside[gap:self.rows - gap] = True
        self.inside = inside
        out = torch.from_numpy(~inside).cuda()
        for t in (self.q, self.k, self.v, self.dout):
            t[out] = float("nan")
        self.row_start = i32(self.start)

    def run(self):
        self.out = torch.full((self.rows, self.H, self.hd), 7.0, dtype=self.dtype, device="cuda")
        self.lse = torch.full((self.rows, self.H), 7.0, device="cuda")
        vla.prompt_attention(self.q, self.k, self.v, self.row_start, self.scale, out=self.out, lse=self.lse)
        return self.out, self.lse

    def back(self):
        K, hd, H = self.K, self.hd, self.H
        g = torch.full((self.rows, (H + 2 * K) * hd + 8), 7.0, dtype=self.dtype, device="cuda")
        self.dq, self.dk, self.dv = (t.unflatten(1, (-1, hd)) for t in g.split([H * hd, K * hd, K * hd, 8], 1)[:3])
        vla.prompt_attention_backward(self.q, self.k, self.v, self.out, self.lse, self.dout, self.row_start, self.scale,
                                      dq=self.dq, dk=self.dk, dv=self.dv)
        assert (g[:, -8:] == 7).all()
        return self.dq, self.dk, self.dv

    def unit_p(self):  # scores: sums of head_dim products in fp32, scaled and taken from the maximum
        return 2 * (self.hd + 32) * U32

    def unit_w(self):
        return torch.finfo(self.dtype).eps / 2

    def check_forward(self, sel=None):
        """Rows of no sequence are left as they were; the others (those of `sel`) agree with the oracle."""
        ref, rlse, mag, smax = po.attention(f64(self.q), f64(self.k), f64(self.v), self.start, self.scale)
        got, lse = f64(self.out), f64(self.lse)
        assert (got[~self.inside] == 7).all() and (lse[~self.inside] == 7).all()
        sel = self.inside if sel is None else sel
        n = np.diff(self.start).max()
        tol = half_step(ref, self.dtype) * (1 + 2 ** -6) + mag * (self.unit_w() + n * U32 + self.unit_p() * np.maximum(smax, 1.0)[..., None])
        bad = (np.abs(got - ref) / tol)[sel]
        assert np.all(bad <= 1), (np.nanmax(bad), np.argwhere(~(bad <= 1))[:5])
        ltol = self.unit_p() * np.maximum(smax, 1.0) + 4 * U32 * np.abs(rlse) + n * U32
        fin = np.isfinite(rlse)
        assert np.array_equal(np.isneginf(lse[sel]), np.isneginf(rlse[sel]))
        assert np.all((np.abs(lse - rlse) <= ltol)[fin & sel[:, None]])
        return bad.max(), tol

    def check_backward(self, sel=None, sel_kv=None):
        """As check_forward, dq at `sel`, dk and dv at `sel_kv`."""
        _, _, mag, smax = po.attention(f64(self.q), f64(self.k), f64(self.v), self.start, self.scale)
        out_err = half_step(np.nan_to_num(f64(self.out)), self.dtype) + mag * (self.unit_w() + 3 * self.unit_p() * np.maximum(smax, 1.0)[..., None])
        # a second exponential, of the score less the log-sum-exp, each with the forward's error
        g, e = po.backward(f64(self.q), f64(self.k), f64(self.v), f64(self.dout), self.start, self.scale, self.unit_w(),
                           3 * self.unit_p(), (self.hd + 32) * U32, out_err)
        worst = 0
        for name, got, ref, err, s in (("dq", self.dq, g[0], e[0], sel), ("dk", self.dk, g[1], e[1], sel_kv),
                                       ("dv", self.dv, g[2], e[2], sel_kv)):
            got, s = f64(got), self.inside if s is None else s
            assert (got[~self.inside] == 7).all(), name
            bad = (np.abs(got - ref) / (half_step(ref, self.dtype) * (1 + 2 ** -6) + err))[s]
            assert np.all(bad <= 1), (name, np.nanmax(bad), np.argwhere(~(bad <= 1))[:5])
            worst = max(worst, bad.max(initial=0))
        return worst

    def both(self, label):
        self.run()
        a = self.check_forward()[0]
        first = [bits(t) for t in self.back()]
        b = self.check_backward()
        assert all(torch.equal(x, bits(y)) for x, y in zip(first, self.back()))  # fixed order of sums
        log(f"[{label}] worst err/tol forward {a:.3f} backward {b:.3f}")


LENS = [[1], [2, 1, 3], [31, 32, 33, 0, 1], [63, 64, 65], [127, 0, 128, 129], [278], [255, 1, 256, 257, 0], [5, 700]]


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("H,K", [(4, 4), (6, 2), (7, 1)])
@pytest.mark.parametrize("hd,dtype", [(64, BF), (128, BF), (128, FP), (256, BF), (64, FP), (256, FP)])
def test_attention_and_gradient(lens, H, K, hd, dtype):
    Case(lens, H, K, hd, dtype, seed=len(lens) + hd, joint=K > 1).both(f"{lens} H={H}/{K} hd={hd} {dtype}")


@pytest.mark.parametrize("hd,dtype", [(64, BF), (128, FP), (128, BF), (256, BF)])
def test_many_workgroups(hd, dtype):
    """Rows enough for each size of workgroup, more sequences than a wave has lanes, empty ones among them."""
    rng = np.random.default_rng(hd)
    for n, most, H in ((200, 40, 8), (70, 300, 8), (3, 900, 32), (5000, 2, 2)):
        lens = rng.integers(0, most + 1, n)
        Case(lens, H, 2, hd, dtype, seed=n, gap=1).both(f"{n} sequences of up to {most}, hd={hd}")


@pytest.mark.parametrize("scale", [-0.3, 0.0, 3.0, 1e-30])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_scales(scale, dtype):
    Case([70, 33], 4, 2, 64, dtype, seed=3, scale=scale, qscale=0.7).both(f"scale {scale}")


@pytest.mark.parametrize("dtype", [BF, FP])
def test_outliers(dtype):
    """One key far above the others, then many small weights; and gradients of very different sizes."""
    c = Case([300, 200], 4, 2, 128, dtype, seed=4)
    c.k[10] *= 6
    c.v[10] *= 30
    c.dout[40:60] *= 100
    c.dout[100:130] *= 1e-3
    c.dout[330:] *= 1e-3
    c.both("outliers")


def test_gradient_sizes_of_half_precision():
    """The whole range: gradients near the smallest normal number, and near the largest."""
    for size, v in ((2e-4, 1.0), (1e-3, 1e-2), (5e4, 0.02), (1e4, 50.0)):
        c = Case([150, 90], 4, 1, 64, FP, seed=6)
        c.dout *= size
        c.v *= v
        if size == 1e4:
            c.q *= 0.05
            c.k *= 0.05
        c.both(f"dout x {size}, v x {v}")


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("what", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("hd,dtype,K", [(64, BF, 2), (128, FP, 1), (128, BF, 2), (256, BF, 2)])
def test_bad_elements_go_no_further_than_the_formulas(what, value, hd, dtype, K):
    """An infinite or NaN element in the middle of a sequence: earlier rows, later keys, other sequences and other key heads
    are what they are without it."""
    lens, H = [40, 150, 33], 4
    for at in (0, 17, 31, 32, 63, 64, 100, 149):
        c = Case(lens, H, K, hd, dtype, seed=at)
        r = int(c.start[1]) + at
        head = {"q": 1, "dout": 1}.get(what, 0)
        getattr(c, what)[r, head, 5] = value
        c.run()
        c.back()
        clean = Case(lens, H, K, hd, dtype, seed=at)
        clean.run()
        clean.back()
        got, tol = f64(c.out), clean.check_forward()[1]
        ref, (dq, dk, dv) = f64(clean.out), (f64(t) for t in (clean.dq, clean.dk, clean.dv))
        rows = np.arange(c.rows)
        hit = (rows >= r) & (rows < int(c.start[2]))           # rows whose formulas hold the key
        heads = np.arange(H) // (H // K) == (head * K // H if what in ("q", "dout") else head)
        if what in ("q", "dout"):
            heads = np.arange(H) == head
            hit = rows == r
        if what != "dout":
            bad = ~(np.abs(got - ref) <= tol)
            assert not bad[~hit & c.inside].any() and not bad[:, ~heads][c.inside].any()
        assert not np.isnan(f64(c.dq)[~hit & c.inside]).any()
        size = np.abs(dq[c.inside]).max()
        assert np.abs(f64(c.dq)[~hit & c.inside] - dq[~hit & c.inside]).max() <= 0.02 * size
        # keys behind the row have nothing of it, nor have other sequences and key heads
        free = (rows > r) | (rows < int(c.start[1])) if what in ("q", "dout") else (rows < int(c.start[1])) | (rows >= int(c.start[2]))
        kv = head * K // H if what in ("q", "dout") else head
        for name, want in (("dk", dk), ("dv", dv)):
            g = f64(getattr(c, name))
            assert np.abs(g - want)[free & c.inside].max() <= 0.02 * np.abs(want[c.inside]).max(), name
            if K > 1:
                assert np.array_equal(g[c.inside][:, 1 - kv], want[c.inside][:, 1 - kv]), name


@pytest.mark.parametrize("hd,dtype", [(64, BF), (128, FP), (256, BF)])
def test_scores_of_minus_infinity(hd, dtype):
    """A key of -inf has no weight; a row that has no other gets zeros and a log-sum-exp of -inf, and gives no gradient."""
    c = Case([100, 40], 4, 2, hd, dtype, seed=9)
    c.q[:, :, 0] = c.q[:, :, 0].abs() + 0.1
    s = int(c.start[0])
    c.k[s:s + 3, :, 0] = -INF
    c.k[s + 70, :, 0] = -INF
    c.run()
    out, lse = f64(c.out), f64(c.lse)
    assert (out[s:s + 3] == 0).all() and np.isneginf(lse[s:s + 3]).all()
    dead = np.zeros(c.rows, bool)
    dead[[s, s + 1, s + 2, s + 70]] = True
    kk, vv = f64(c.k), f64(c.v)
    keep = c.inside & ~dead
    for h in range(4):  # the oracle over the keys that are left
        for a, n in ((s, 100), (int(c.start[1]), 40)):
            for i in range(a, a + n):
                js = [j for j in range(a, i + 1) if not dead[j]]
                if not js:
                    continue
                o, z, mag, smax = co.attention(f64(c.q)[i, h], kk[js, h // 2], vv[js, h // 2], c.scale)
                tol = half_step(o, dtype) * 1.02 + mag * (c.unit_w() + 100 * U32 + c.unit_p() * max(smax, 1))
                assert np.all(np.abs(out[i, h] - o) <= tol) and abs(z - lse[i, h]) <= c.unit_p() * max(smax, 1) + 1e-5
    c.back()
    dv = f64(c.dv)
    assert np.isfinite(dv[c.inside]).all() and (dv[dead] == 0).all() and (dv[keep] != 0).any()
    assert (f64(c.dq)[s:s + 3, :, 1:] == 0).all()


def test_infinite_scores_are_nan_rows():
    c = Case([40], 2, 2, 64, BF, seed=2)
    s = int(c.start[0])
    c.q[s + 20, 0, 0], c.k[s + 3, 0, 0] = 1.0, INF
    c.q[s:s + 20, 0, 0] = 1.0
    c.run()
    assert np.isnan(f64(c.out)[s + 20, 0]).all() and np.isfinite(f64(c.out)[s:s + 3]).all() and np.isfinite(f64(c.out)[:, 1]).all()


@pytest.mark.parametrize("start", [[4, 2, 9, 30], [-3, 5, 9], [0, 10, 200], [200, 300], [7, 7, 7], [30, 20, 10, 0], [0, 2 ** 31 - 1, 10, 12],
                                   [-2 ** 31, 2 ** 31 - 1]], ids=str)
def test_bounds_outside_are_passed_over(start):
    """Sequences whose bounds descend or lie outside are not read nor written; the others are."""
    rows, H, K, hd = 40, 2, 1, 64
    q, k, v, do = rand((rows, H, hd), BF, 1), rand((rows, K, hd), BF, 2), rand((rows, K, hd), BF, 3), rand((rows, H, hd), BF, 4)
    t = i32(start)
    lse = torch.full((rows, H), 7.0, device="cuda")
    out = torch.full((rows, H, hd), 7.0, dtype=BF, device="cuda")
    vla.prompt_attention(q, k, v, t, 0.1, out=out, lse=lse)
    g = [torch.full(x.shape, 7.0, dtype=BF, device="cuda") for x in (q, k, v)]
    vla.prompt_attention_backward(q, k, v, out, lse, do, t, 0.1, dq=g[0], dk=g[1], dv=g[2])
    seqs = po.sequences(start, rows)
    within = np.zeros(rows, bool)
    for a, n in seqs:
        within[a:a + n] = True
    for x in (out, *g):
        assert (f64(x)[~within] == 7).all()
    ascending = all(a <= b for a, b in zip(start, start[1:]))
    if ascending and seqs:
        ref = po.attention(f64(q), f64(k), f64(v), start, 0.1)[0]
        assert np.abs(f64(out) - ref)[within].max() < 0.02 and (f64(out)[within] != 7).any()


def test_rows_far_into_a_large_buffer():
    """Element offsets past 2^31: the last rows of a projection as wide as they come."""
    ld, rows, H, K, hd = 1 << 17, 17000, 4, 2, 64
    x = torch.zeros((rows, ld), dtype=BF, device="cuda")
    start = [rows - 90, rows - 60, rows]
    part = rand((90, (H + 2 * K) * hd), BF, 5)
    x[-90:, ld - (H + 2 * K) * hd:] = part
    q, k, v = (t.unflatten(1, (-1, hd)) for t in x[:, ld - (H + 2 * K) * hd:].split([H * hd, K * hd, K * hd], 1))
    lse = torch.empty((rows, H), device="cuda")
    out = vla.prompt_attention(q, k, v, i32(start), 0.2, lse=lse)
    do = torch.zeros((rows, H, hd), dtype=BF, device="cuda")
    do[-90:] = rand((90, H, hd), BF, 6)
    g = vla.prompt_attention_backward(q, k, v, out, lse, do, i32(start), 0.2)
    small = [t.unflatten(1, (-1, hd)) for t in part.split([H * hd, K * hd, K * hd], 1)]
    ss, slse = i32([0, 30, 90]), torch.empty((90, H), device="cuda")
    sout = vla.prompt_attention(*small, ss, 0.2, lse=slse)
    assert torch.equal(sout, out[-90:]) and torch.equal(slse, lse[-90:])
    again = vla.prompt_attention_backward(*small, sout, slse, do[-90:], ss, 0.2)
    assert torch.equal(again[0], g[0][-90:])
    # the keys' sums may be split otherwise among as many rows: two results within the same bound of the formulas'
    c = Case.__new__(Case)
    c.hd, c.dtype = hd, BF
    x64 = [f64(t) for t in small]
    _, _, mag, smax = po.attention(*x64, [0, 30, 90], 0.2)
    out_err = half_step(f64(sout), BF) + mag * (c.unit_w() + 3 * c.unit_p() * np.maximum(smax, 1.0)[..., None])
    ref, err = po.backward(*x64, f64(do[-90:]), [0, 30, 90], 0.2, c.unit_w(), 3 * c.unit_p(), (hd + 32) * U32, out_err)
    for i in (1, 2):
        for got in (again[i], g[i][-90:]):
            assert np.all(np.abs(f64(got) - ref[i]) <= half_step(ref[i], BF) * (1 + 2 ** -6) + err[i])


def test_single_rows_and_none():
    c = Case([1, 1, 0, 1], 4, 2, 128, BF, seed=8)
    c.both("single rows")
    for h in range(4):
        assert torch.equal(c.out[torch.from_numpy(c.inside).cuda(), h], c.v[torch.from_numpy(c.inside).cuda(), h // 2])
    q = torch.empty((0, 4, 128), dtype=BF, device="cuda")
    kv = torch.empty((0, 2, 128), dtype=BF, device="cuda")
    assert vla.prompt_attention(q, kv, kv, i32([0, 0]), 0.1).shape == (0, 4, 128)
    e = torch.full((3, 4, 128), 7.0, dtype=BF, device="cuda")
    x = rand((3, 4, 128), BF, 1)
    assert (vla.prompt_attention(x, x, x, i32([0]), 0.1, out=e) == 7).all()


def test_streams_and_graphs():
    """Two streams at once, each with its own buffers, and a captured forward and backward replayed on new inputs beside
    eager work: the same bits as eager calls."""
    a, b = Case([200, 77, 300], 8, 2, 128, BF, seed=1), Case([30, 400], 4, 4, 64, FP, seed=2)
    want = []
    for c in (a, b):
        c.run()
        c.back()
        want.append([bits(t).clone() for t in (c.out, c.dq, c.dk, c.dv)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, c in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                c.run()
                c.back()
        torch.cuda.synchronize()
        for c, w in zip((a, b), want):
            assert all(torch.equal(bits(t), x) for t, x in zip((c.out, c.dq, c.dk, c.dv), w))
    ws = vla.prompt_attention_backward_workspace(a.q, a.k, a.row_start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vla.prompt_attention(a.q, a.k, a.v, a.row_start, a.scale, out=a.out, lse=a.lse)
        vla.prompt_attention_backward(a.q, a.k, a.v, a.out, a.lse, a.dout, a.row_start, a.scale, dq=a.dq, dk=a.dk, dv=a.dv, workspace=ws)
    for seed in (5, 6, 7):
        n = Case([200 - seed, 77 + seed, 300], 8, 2, 128, BF, seed=seed)  # as many rows, other lengths
        n.run()
        n.back()
        for x, y in ((a.q, n.q), (a.k, n.k), (a.v, n.v), (a.dout, n.dout), (a.row_start, n.row_start)):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for t in ("out", "dq", "dk", "dv"):
            assert torch.equal(bits(getattr(a, t)), bits(getattr(n, t))), t
        b.run()


def test_norm_rope_attention_and_their_gradients_together():
    """A decoder layer's attention over a packed batch, as training runs it: plan's row_start, head norms and rotation,
    attention, and back through both; against the composed oracle."""
    H, K, hd, lens, eps = 6, 2, 64, [40, 1, 97], 1e-6
    rows = sum(lens)
    n = len(lens)
    plan = vla.kv_plan(i32([0] * n), i32(lens), i32(np.full((n, 9), -1)), i32(range(40)), 40, rows)
    qkv = rand((rows, (H + 2 * K) * hd), BF, 1)
    q, k, v = (t.unflatten(1, (-1, hd)) for t in qkv.split([H * hd, K * hd, K * hd], 1))
    gains = [(1 + rand((hd,), torch.float32, s, 0.2)).to(BF) for s in (2, 3)]
    freqs, _ = vla.rope_freqs(hd)
    scale = hd ** -0.5
    qr, kr = vla.qk_norm_rope(q, k, plan["row_pos"], freqs, *gains, eps)
    lse = torch.empty((rows, H), device="cuda")
    out = vla.prompt_attention(qr, kr, v, plan["row_start"], scale, lse=lse)
    dout = rand((rows, H, hd), BF, 5)
    dqr, dkr, dv = vla.prompt_attention_backward(qr, kr, v, out, lse, dout, plan["row_start"], scale)
    dq, dk, dgq, dgk = vla.qk_norm_rope_backward(q, k, dqr, dkr, plan["row_pos"], freqs, *gains, eps)
    # the oracle of the whole, in 64 bits
    pos = plan["row_pos"].cpu().numpy()
    start = plan["row_start"].cpu().numpy()
    fr = f64(freqs)
    tq, tk = (co.norm_turn(f64(x), f64(g), eps, pos, fr, "half") for x, g in ((q, gains[0]), (k, gains[1])))
    ref = po.attention(tq, tk, f64(v), start, scale)[0]
    (gq, gk, gv), _ = po.backward(tq, tk, f64(v), f64(dout), start, scale)
    want = [ref, gv]
    for x, g, d in ((q, gains[0], gq), (k, gains[1], gk)):
        want += list(co.norm_turn_backward(f64(x), f64(g), eps, pos, fr, "half", d))
    for name, got, w in zip(("out", "dv", "dq", "dq_gain", "dk", "dk_gain"), (out, dv, dq, dgq, dk, dgk), want):
        # q, k, out, dq and dk are rounded to bf16 (2^-9 of each) between the steps, weights once in each product
        err = np.linalg.norm(f64(got) - w) / np.linalg.norm(w)
        assert err < 8 * 2.0 ** -9, (name, err)
