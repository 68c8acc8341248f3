"""Host-side checks of the cache in 8-bit numbers (vla_cache.h): pins of its oracle, and the refusals, all of which come before
any device work."""
import math

import numpy as np
import pytest

from oracle import cache_f8_oracle as c8
from test_cache_host import P, _call, _each, vla  # noqa: F401  (a fixture)


# ------------------------------------------------------------------ oracle pins
def test_numbers_are_torchs():
    import torch
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, c8.NUMBERS, equal_nan=True)
    assert c8.NUMBERS[0x7e] == 448 and c8.NUMBERS[1] == 2.0 ** -9


def test_encode_worked_by_hand():
    """The largest becomes 448; 17 / 16 lies half way between 1 and 18 / 16 and goes to the even one, as 19 / 16 does."""
    x = np.array([[448.0, 1.0, 17 / 16, 19 / 16, -2.0 ** -10, 2.0 ** -10 * 1.01, 0.0, 300.0]])
    b, s = c8.encode(x)
    assert s[0] == 1.0 and c8.NUMBERS[b[0]].tolist() == [448, 1, 1, 20 / 16, 0, 2.0 ** -9, 0, 288]
    b, s = c8.encode(np.array([[7.0, 17 / 64, -19 / 64]]))  # the same numbers times 1 / 64
    assert c8.NUMBERS[b[0]].tolist() == [448, 16, -20] and s[0] == np.float32(7 / 448)


def test_encode_error_bound():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(200, 64)) * np.exp(rng.normal(size=(200, 64)) * 3)
    b, s = c8.encode(x)
    unit = np.abs(x).max(-1, keepdims=True) / 448
    assert np.all(np.abs(c8.NUMBERS[b] * unit - x) <= np.maximum(np.abs(x) * 2.0 ** -4, unit * 2.0 ** -10) * (1 + 1e-12))


def test_encode_zeros_and_not_finite():
    b, s = c8.encode(np.array([[0.0, 0.0], [1.0, np.inf], [np.nan, 0.0], [2.0 ** -110, 0.0]]))
    assert b[0].tolist() == [0, 0] and s[0] == np.float32(c8.LEAST / 448) and np.isnan(s[1:3]).all()
    assert np.isnan(c8.NUMBERS[b[1:3]]).all() and c8.NUMBERS[b[3, 0]] == 448 * 2.0 ** -10


# ------------------------------------------------------------------ refusals
SIZES = [(-1, dict(rows=-1)), (-1, dict(kv=0)), (-7, dict(kv=2000)), (-7, dict(hd=96)), (-7, dict(dtype=2)), (-1, dict(n_pages=-1)),
         (-7, dict(n_pages=1 << 27)), (-7, dict(rows=2 ** 31 - 1, kv=1024, ld_k=1 << 20, ld_v=1 << 20))]
TENSORS = [(-1, {x: None}) for x in ("k", "v", "kp", "vp", "ks", "vs", "slot")] + [
    (-1, dict(k=P + 8)), (-1, dict(v=P + 2)), (-1, dict(ld_k=248)), (-1, dict(ld_v=260)), (-1, dict(kp=P + 8)), (-1, dict(vp=P + 1))]


def test_append_refusals(vla):  # noqa: F811
    good = dict(rows=4, kv=2, hd=128, dtype=0, k=P, ld_k=256, v=P, ld_v=256, kp=P, vp=P, ks=P, vs=P, n_pages=3, slot=P, stream=None)
    _each(vla, "vla_kv_append_f8", good, SIZES + TENSORS)
    assert _call(vla, "vla_kv_append_f8", good, rows=0, k=None, slot=None)[0] == 0


def test_read_refusals(vla):  # noqa: F811
    good = dict(rows=4, kv=2, hd=128, dtype=1, kp=P, vp=P, ks=P, vs=P, n_pages=3, slot=P, k=P, ld_k=256, v=P, ld_v=256, stream=None)
    _each(vla, "vla_kv_read_f8", good, SIZES + TENSORS)
    assert _call(vla, "vla_kv_read_f8", good, rows=0, k=None, slot=None)[0] == 0


def test_attention_refusals(vla):  # noqa: F811
    good = dict(n_env=4, heads=8, kv=2, hd=128, dtype=0, q=P, ld_q=1024, kp=P, vp=P, ks=P, vs=P, n_pages=9, table=P, ld=8,
                max_pages=8, lens=P, scale=0.1, out=2 * P, ld_o=1024, lse=None, ws=P, bytes=1 << 40, stream=None)
    _each(vla, "vla_paged_attention_f8", good, [
        (-1, dict(n_env=-1)), (-7, dict(n_env=1 << 16)), (-1, dict(kv=3)), (-7, dict(hd=80)), (-7, dict(dtype=2)), (-1, dict(n_pages=-1)),
        (-1, dict(scale=math.nan)), (-1, dict(q=None)), (-1, dict(out=None)), (-1, dict(ld_q=8)), (-1, dict(ld=7)),
        (-1, dict(table=None)), (-1, dict(lens=None)), (-1, dict(kp=None)), (-1, dict(vp=None)), (-1, dict(ks=None)),
        (-1, dict(vs=None)), (-1, dict(kp=P + 8)), (-3, dict(ws=None)), (-3, dict(bytes=0)), (-3, dict(ws=P + 16))])
    assert _call(vla, "vla_paged_attention_f8", good, n_env=0, q=None, out=None, ws=None)[0] == 0


def test_binding_refuses(vla):  # noqa: F811
    import torch
    t, i = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    f8, s = torch.zeros(3, 4, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(3, 4, 16)
    for call in (lambda: vla.kv_append_f8(t, t, i, f8, f8.transpose(2, 3).contiguous(), s, s),
                 lambda: vla.kv_read_f8(i, f8, f8.transpose(2, 3).contiguous(), s, s),
                 lambda: vla.paged_attention_f8(t, f8, f8.transpose(2, 3).contiguous(), s, s, i[:, None], i, 0.1)):
        with pytest.raises(ValueError):
            call()
