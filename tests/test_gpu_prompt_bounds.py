"""Attention over whole prompts and its gradient beside sequences whose bounds descend or lie outside the tensors: those are
passed over, the others are what the formulas say, in every pass, wherever the bad bounds stand."""
import numpy as np
import pytest
import torch

from gpu_util import log
from oracle import prompt_oracle as po
from paper_2505_18719_amd import vla
from test_gpu_cache import BF, FP, f64, i32, rand
from test_gpu_prompt import Case

pytestmark = pytest.mark.gpu

FAR = 2 ** 31 - 1


class Bounds(Case):
    """A row_start as it comes; rows of no sequence are NaN in the inputs, and the gradient's workspace is NaN beforehand."""

    def __init__(self, row_start, rows, H, K, hd, dtype, seed=0):
        seqs = po.sequences(row_start, rows)
        ends = sorted((a, a + n) for a, n in seqs)
        assert all(b <= c for (_, b), (c, _) in zip(ends, ends[1:]))  # no shared rows
        self.rows, self.H, self.K, self.hd, self.dtype, self.scale = rows, H, K, hd, dtype, hd ** -0.5
        self.start = np.array([x for e in ends for x in e], np.int64)  # what lies between two of them is not looked at
        self.inside = np.zeros(rows, bool)
        for a, b in ends:
            self.inside[a:b] = True
        self.q, self.k, self.v, self.dout = (rand((rows, h, hd), dtype, seed + i, s)
                                             for i, (h, s) in enumerate(((H, 2.0), (K, 1.0), (K, 1.0), (H, 0.1))))
        out = torch.from_numpy(~self.inside).cuda()
        for t in (self.q, self.k, self.v, self.dout):
            t[out] = float("nan")
        self.row_start = i32(row_start)

    def back(self):
        g = [torch.full(x.shape, 7.0, dtype=self.dtype, device="cuda") for x in (self.q, self.k, self.v)]
        ws = vla.prompt_attention_backward_workspace(self.q, self.k, self.row_start).fill_(255)
        self.dq, self.dk, self.dv = vla.prompt_attention_backward(
            self.q, self.k, self.v, self.out, self.lse, self.dout, self.row_start, self.scale, dq=g[0], dk=g[1], dv=g[2], workspace=ws)
        return self.dq, self.dk, self.dv


@pytest.mark.parametrize("start,rows", [([400, 2, 900, 1300], 1300), ([0, 640, -3, 1280, 1920], 2000), ([0, 10, FAR, 12, 500], 1000),
                                        ([700, 1200, 5, 600, -1, 650, 690], 1250), ([-2 ** 31, 100, 300, 5000, 301, 302], 400),
                                        ([1500, 1500, 900, 1400, 300, 800, 0, 290], 1500), ([-1, 0, FAR, 0, 333], 333)], ids=str)
@pytest.mark.parametrize("H,K,hd,dtype", [(4, 1, 64, BF), (2, 2, 64, FP), (16, 8, 64, BF), (4, 2, 128, FP), (2, 2, 256, BF)])
def test_bad_bounds_between_sequences(start, rows, H, K, hd, dtype):
    Bounds(start, rows, H, K, hd, dtype, seed=rows).both(f"{start} H={H}/{K} hd={hd} {dtype}")


@pytest.mark.parametrize("n", [63, 64, 65, 130, 448, 512])
@pytest.mark.parametrize("H,K,hd,dtype", [(4, 2, 64, BF), (6, 1, 128, FP), (2, 2, 256, BF)])
def test_bad_bounds_among_many(n, H, K, hd, dtype):
    """Every seventh bound or so is bad, of sequences of 0 to 20 rows with one of 700 in between: each costs two of them."""
    rng = np.random.default_rng(n + hd)
    lens = rng.integers(0, 21, n)
    lens[n // 3] = 700
    start = np.concatenate([[0], np.cumsum(lens)]) + 3
    rows = int(start[-1]) + 5
    bad = rng.random(n + 1) < 1 / 7
    bad[[n // 3, n // 3 + 1]] = False
    start[bad] = rng.choice([-1, -2 ** 31, rows + 1, FAR], bad.sum())
    Bounds(start, rows, H, K, hd, dtype, seed=n).both(f"{n} sequences, {int(bad.sum())} bad bounds, hd={hd}")


def test_more_sequences_than_are_listed():
    """Of 600 sequences the bounds do not ascend: their rows' values are left open, other rows' are as they were."""
    rows, n, H, K, hd = 3000, 600, 2, 1, 64
    for start in ([-1] + [2000 + 10 * s for s in range(1, 7)] + [0] * 594, [0] * 300 + [2500, 2510, -5] + [1] * 298,
                  [FAR] + list(range(2900, 2300, -1))):
        assert len(start) == n + 1
        c = Bounds(start, rows, H, K, hd, BF)
        c.run()
        c.back()
        for t in (c.out, c.lse, c.dq, c.dk, c.dv):
            assert (f64(t)[~c.inside] == 7).all()
    log("600 sequences")
