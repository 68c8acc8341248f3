"""Host-side checks of attention over whole prompts (vla_prompt.h): pins of its oracle, and the refusals, all of which come
before any device work."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import prompt_oracle as po

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def vla():
    from paper_2505_18719_amd import vla as binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2505_18719_amd import build
        build.build(verbose=False)
    binding.load_library()
    return binding


@pytest.mark.parametrize("lang", ["c", "c++"])
def test_header_compiles_on_its_own(lang, tmp_path):
    cc = shutil.which("gcc" if lang == "c" else "g++")
    if cc is None:
        pytest.skip("no host compiler")
    src = tmp_path / ("h.c" if lang == "c" else "h.cpp")
    src.write_text('#include "vla_prompt.h"\nint main(void) { return 0; }\n')
    std = ["-std=c99", "-pedantic"] if lang == "c" else ["-std=c++17"]
    r = subprocess.run([cc, *std, "-Wall", "-Wextra", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"),
                        str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


# ------------------------------------------------------------------ oracle pins
def test_attention_worked_by_hand():
    """Two sequences; equal scores weigh alike, and a score ln 3 larger weighs three times as much."""
    q = np.array([[[1.0]], [[1.0]], [[2.0]], [[1.0]]])
    k = np.array([[[0.0]], [[math.log(3)]], [[5.0]], [[5.0]]])
    v = np.array([[[4.0]], [[8.0]], [[1.0]], [[3.0]]])
    out, lse, _, _ = po.attention(q, k, v, [0, 2, 4], 1.0)
    assert np.allclose(out[:, 0, 0], [4, 7, 1, 2])
    assert np.allclose(lse[:, 0], [0, math.log(4), 10, 5 + math.log(2)])


def test_heads_share_keys_in_order():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(5, 6, 4)), rng.normal(size=(5, 2, 4)), rng.normal(size=(5, 2, 4))
    out = po.attention(q, k, v, [0, 5], 0.7)[0]
    wide = po.attention(q, np.repeat(k, 3, 1), np.repeat(v, 3, 1), [0, 5], 0.7)[0]
    assert np.allclose(out, wide)


@pytest.mark.parametrize("scale", [0.4, -0.9])
def test_gradient_against_differences(scale):
    rng = np.random.default_rng(3)
    x = [rng.normal(size=(7, h, 3)) for h in (4, 2, 2)]
    dout = rng.normal(size=(7, 4, 3))
    start = [0, 4, 4, 7]
    g, _ = po.backward(*x, dout, start, scale)

    def loss():
        return (po.attention(*x, start, scale)[0] * dout).sum()
    for t, dt in zip(x, g):
        for i in rng.integers(0, t.size, 12):
            was = t.flat[i]
            t.flat[i] = was + 1e-5
            up = loss()
            t.flat[i] = was - 1e-5
            down = loss()
            t.flat[i] = was
            assert abs((up - down) / 2e-5 - dt.flat[i]) < 1e-8


def test_rows_of_no_sequence():
    assert po.sequences([2, 5, 5, 3, 9, 12], 10) == [(2, 3), (3, 6)]
    assert po.sequences([-1, 4, 6], 6) == [(4, 2)]


# ------------------------------------------------------------------ refusals
P = 1 << 20  # an aligned address that is never read: the checks fail first


def _call(vla, name, good, **change):
    args = dict(good, **change)
    rc = getattr(vla.load_library(), name)(*args.values())
    return rc, vla.load_library().vla_last_error()


def _each(vla, name, good, refusals):
    for code, change in refusals:
        rc, msg = _call(vla, name, good, **change)
        assert rc == code and msg, (name, change, rc, msg)


SIZES = [(-1, dict(rows=-1)), (-1, dict(n_seq=-1)), (-1, dict(heads=0)), (-1, dict(kv=0)), (-1, dict(kv=3)), (-7, dict(heads=2000)),
         (-7, dict(hd=96)), (-7, dict(hd=32)), (-7, dict(dtype=2)), (-7, dict(dtype=-1)), (-7, dict(n_seq=1 << 26)),
         (-7, dict(rows=2 ** 31 - 1, heads=1024, kv=1)), (-1, dict(scale=math.nan)), (-1, dict(scale=math.inf)), (-1, dict(scale=3e38))]


def test_forward_refusals(vla):
    good = dict(rows=4, n_seq=2, heads=8, kv=2, hd=128, dtype=0, q=P, ld_q=1024, k=2 * P, ld_k=256, v=3 * P, ld_v=256, start=P,
                scale=0.1, out=4 * P, ld_o=1024, lse=None, stream=None)
    _each(vla, "vla_prompt_attention", good, SIZES + [
        (-1, dict(q=None)), (-1, dict(k=None)), (-1, dict(v=None)), (-1, dict(out=None)), (-1, dict(start=None)),
        (-1, dict(q=P + 2)), (-1, dict(v=3 * P + 8)), (-1, dict(ld_q=1016)), (-1, dict(ld_q=1028)), (-1, dict(ld_k=0)),
        (-1, dict(ld_o=8)), (-1, dict(ld_v=-256)), (-7, dict(ld_k=(1 << 23) + 8)), (-1, dict(out=P)), (-1, dict(out=2 * P)),
        (-1, dict(out=3 * P)), (-1, dict(out=P + 1024)), (-1, dict(q=P, ld_q=2048, out=P + 2 * 1016, ld_o=2048)),
        (-1, dict(out=2 * P - 16, ld_o=1024))])
    assert _call(vla, "vla_prompt_attention", good, rows=0, q=None, k=None, v=None, out=None)[0] == 0
    assert _call(vla, "vla_prompt_attention", good, n_seq=0, q=None, start=None)[0] == 0


def test_backward_refusals(vla):
    good = dict(rows=4, n_seq=2, heads=8, kv=2, hd=64, dtype=1, q=P, ld_q=512, k=2 * P, ld_k=128, v=3 * P, ld_v=128, out=4 * P,
                ld_o=512, lse=P, dout=5 * P, ld_do=512, start=P, scale=0.1, dq=6 * P, ld_dq=512, dk=7 * P, ld_dk=128, dv=8 * P,
                ld_dv=128, ws=9 * P, bytes=1 << 30, stream=None)
    _each(vla, "vla_prompt_attention_backward", good, SIZES + [
        (-1, {x: None}) for x in ("q", "k", "v", "out", "lse", "dout", "start", "dq", "dk", "dv")] + [
        (-1, dict(dq=P)), (-1, dict(dq=5 * P)), (-1, dict(dk=2 * P)), (-1, dict(dv=3 * P)), (-1, dict(dv=7 * P)), (-1, dict(dk=6 * P)),
        (-1, dict(dq=4 * P)), (-1, dict(ld_dq=504)), (-1, dict(ld_do=508)), (-1, dict(dout=5 * P + 8)), (-7, dict(ld_dv=1 << 24)),
        (-3, dict(ws=None)), (-3, dict(bytes=64)), (-3, dict(ws=9 * P + 16))])
    assert _call(vla, "vla_prompt_attention_backward", good, rows=0, q=None, ws=None)[0] == 0
    assert _call(vla, "vla_prompt_attention_backward", good, n_seq=0, q=None, ws=None)[0] == 0
    n = ctypes.c_size_t()
    lib = vla.load_library()
    assert lib.vla_prompt_attention_backward_workspace_size(100, 3, 8, 2, 64, ctypes.byref(n)) == 0 and n.value >= 6400
    assert lib.vla_prompt_attention_backward_workspace_size(100, 3, 8, 3, 64, ctypes.byref(n)) == -1
    assert lib.vla_prompt_attention_backward_workspace_size(100, 3, 8, 2, 64, None) == -1


def test_parts_of_one_projection_do_not_overlap(vla):
    """Gradients may be parts of one buffer, as q, k and v are: only what the checks after that refuse is left."""
    good = dict(rows=4, n_seq=2, heads=8, kv=2, hd=64, dtype=1, q=P, ld_q=768, k=P + 1024, ld_k=768, v=P + 1280, ld_v=768,
                out=4 * P, ld_o=512, lse=P, dout=5 * P, ld_do=512, start=P, scale=0.1, dq=6 * P, ld_dq=768, dk=6 * P + 1024,
                ld_dk=768, dv=6 * P + 1280, ld_dv=768, ws=None, bytes=0, stream=None)
    assert _call(vla, "vla_prompt_attention_backward", good)[0] == -3
    assert _call(vla, "vla_prompt_attention_backward", good, dk=6 * P + 1016)[0] == -1


def test_binding_refuses(vla):
    import torch
    t = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: vla.prompt_attention(t, t, t, i, 0.1),
                 lambda: vla.prompt_attention_backward(t, t, t, t, torch.zeros(2, 4), t, i, 0.1)):
        with pytest.raises(ValueError):
            call()
