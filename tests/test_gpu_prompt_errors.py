"""Errors of the gradient of attention over whole prompts as a whole: what its roundings make of it and no more.

The limits are relative errors against the 64-bit oracle, in units of half a step of the type.  They lie between what the kernel's
roundings, taken one by one in 64 bits with these lengths and distributions, make together, and what they make when one of its measures
is left out (one rounding of an output by itself: 0.42 to 0.44):
                                           sequences of up to 5 rows     of 279 rows
    dq  as it is                           0.43                          0.43
        D not exact for the first rows     0.87                          0.51 to 0.55
        dS as one number of the type       0.60                          0.60
    dk  as it is                           0.60                          0.59 to 0.60
        D with the rounding of the output  0.97                          0.65 to 0.68
    dv  as it is                           0.51 to 0.52                  0.58 to 0.59
"""
import numpy as np
import pytest
import torch

from gpu_util import log
from oracle import prompt_oracle as po
from test_gpu_cache import BF, FP, f64
from test_gpu_prompt import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd,dtype", [(64, BF), (128, BF), (256, BF), (64, FP), (128, FP), (256, FP)])
@pytest.mark.parametrize("lens,limits", [([2, 3, 4, 5] * 40, (0.5, 0.75, 0.56)), ([279] * 3, (0.47, 0.63, 0.62))], ids=["short", "279"])
def test_gradient_errors(lens, limits, hd, dtype):
    c = Case(lens, 4, 2, hd, dtype, seed=hd, qscale=1.0)
    c.run()
    c.back()
    want, _ = po.backward(f64(c.q), f64(c.k), f64(c.v), f64(c.dout), c.start, c.scale)
    errs = [np.linalg.norm((f64(x) - w)[c.inside]) / np.linalg.norm(w[c.inside]) / (torch.finfo(dtype).eps / 2)
            for x, w in zip((c.dq, c.dk, c.dv), want)]
    log(f"[{len(lens)} sequences, hd={hd} {dtype}] dq {errs[0]:.3f} dk {errs[1]:.3f} dv {errs[2]:.3f} of half a step")
    assert all(e <= most for e, most in zip(errs, limits)), errs
