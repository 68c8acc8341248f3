"""Host-side checks of attention over shared pages (vla_cache.h): the refusals, all of which come before any device work."""
import ctypes
import math

import pytest

from test_cache_host import P, _call, _each, vla  # noqa: F401  (a fixture)


def test_refusals(vla):  # noqa: F811
    good = dict(n_env=4, n_groups=2, heads=8, kv=2, hd=128, dtype=0, q=P, ld_q=1024, kp=P, vp=P, n_pages=9, table=P, ld=8,
                max_pages=8, lens=P, start=P, shared=P, scale=0.1, out=2 * P, ld_o=1024, lse=None, ws=P, bytes=1 << 40, stream=None)
    _each(vla, "vla_shared_attention", good, [
        (-1, dict(n_env=-1)), (-7, dict(n_env=1 << 16)), (-1, dict(n_groups=-1)), (-7, dict(n_groups=1 << 16)), (-1, dict(max_pages=-1)),
        (-7, dict(max_pages=1 << 26, ld=1 << 26)), (-1, dict(kv=3)), (-1, dict(kv=0)), (-7, dict(hd=80)), (-7, dict(dtype=2)),
        (-1, dict(n_pages=-1)), (-7, dict(n_pages=1 << 27)), (-1, dict(scale=math.nan)), (-1, dict(q=None)), (-1, dict(out=None)),
        (-1, dict(ld_q=8)), (-1, dict(ld_o=1000)), (-1, dict(ld=7)), (-1, dict(table=None)), (-1, dict(lens=None)),
        (-1, dict(kp=None)), (-1, dict(vp=None)), (-1, dict(start=None)), (-1, dict(shared=None)), (-1, dict(kp=P + 8)),
        (-3, dict(ws=None)), (-3, dict(bytes=0)), (-3, dict(ws=P + 16))])
    assert _call(vla, "vla_shared_attention", good, n_env=0, q=None, out=None, ws=None)[0] == 0
    n = ctypes.c_size_t()
    lib = vla.load_library()
    assert lib.vla_shared_attention_workspace_size(4, 2, 8, 2, 128, 8, ctypes.byref(n)) == 0 and n.value > 0
    assert lib.vla_shared_attention_workspace_size(4, 2, 8, 3, 128, 8, ctypes.byref(n)) == -1
    assert lib.vla_shared_attention_workspace_size(4, 2, 8, 2, 128, 8, None) == -1


def test_binding_refuses(vla):  # noqa: F811
    import torch
    t, i = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        vla.shared_attention(t, t[None], t[None], i[:, None], i, i, i[:1], 0.1)
