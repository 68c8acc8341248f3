"""Host-side checks of the paged cache's operators (vla_cache.h): pins of their oracle, the rotation frequencies, and the
refusals, all of which come before any device work."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import cache_oracle as co

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
    src.write_text('#include "vla_cache.h"\nint main(void) { return 0; }\n')
    std = ["-std=c99", "-pedantic"] if lang == "c" else ["-std=c++17"]
    r = subprocess.run([cc, *std, "-Wall", "-Wextra", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"),
                        str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


# ------------------------------------------------------------------ oracle pins
def test_plan_worked_by_hand():
    """Three environments: one with an open page, one new, one whose pages the free list no longer holds, and after it one
    that needs none and is served."""
    table = np.full((4, 3), -1)
    table[0, :2] = [7, 3]
    table[3, 0] = 5
    out, after = co.kv_plan([20, 0, 16, 2], [13, 17, 1, 3], table, [9, 8, 4], 10, 40)
    assert out["lens"].tolist() == [33, 17, 16, 5]
    assert out["row_start"].tolist() == [0, 13, 30, 31, 34]
    assert after.tolist() == [[7, 3, 9], [8, 4, -1], [-1, -1, -1], [5, -1, -1]]
    assert out["row_slot"][:13].tolist() == [3 * 16 + i for i in range(4, 16)] + [9 * 16]
    assert out["row_slot"][13:31].tolist() == [8 * 16 + i for i in range(16)] + [4 * 16, -1]
    assert out["row_slot"][31:].tolist() == [5 * 16 + 2, 5 * 16 + 3, 5 * 16 + 4] + [-1] * 6
    assert out["row_env"][29:35].tolist() == [1, 2, 3, 3, 3, -1]
    assert out["row_pos"][12:14].tolist() == [32, 0]
    assert out["stats"].tolist() == [3, 34, 1]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_depends_on_distance_only_and_keeps_length(layout):
    rng = np.random.default_rng(0)
    f, _ = co.rope_freqs(8, 100.0)
    q, k = rng.normal(size=(1, 1, 12)), rng.normal(size=(1, 1, 12))

    def score(i, j):
        return float((co.turn(q, [i], f, layout) * co.turn(k, [j], f, layout)).sum())
    assert score(5, 3) == pytest.approx(score(105, 103), abs=1e-12)
    y = co.turn(q, [9], f, layout)
    assert (y ** 2).sum() == pytest.approx((q ** 2).sum()) and np.array_equal(y[..., 8:], q[..., 8:])
    a, b = (0, 4) if layout == "half" else (0, 1)  # the first pair turns by one radian per position
    assert y[0, 0, a] == pytest.approx(q[0, 0, a] * math.cos(9) - q[0, 0, b] * math.sin(9))


def test_backward_against_differences():
    rng = np.random.default_rng(1)
    f, _ = co.rope_freqs(8, 50.0)
    x, g, d = rng.normal(size=(3, 2, 12)), 1 + 0.3 * rng.normal(size=12), rng.normal(size=(3, 2, 12))
    pos, h = [0, 4, 77], 1e-6

    def loss(x, g):
        return float((co.norm_turn(x, g, 1e-2, pos, f, "interleaved", 1.3) * d).sum())
    dx, dg = co.norm_turn_backward(x, g, 1e-2, pos, f, "interleaved", d, 1.3)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        assert (loss(x + e, g) - loss(x - e, g)) / (2 * h) == pytest.approx(dx[i], abs=1e-7)
    for i in range(12):
        e = np.zeros_like(g)
        e[i] = h
        assert (loss(x, g + e) - loss(x, g - e)) / (2 * h) == pytest.approx(dg[i], abs=1e-7)


def test_attention_closed_forms():
    v = np.arange(12.0).reshape(4, 3)
    out, lse, mag, _ = co.attention(np.zeros(3), np.ones((4, 3)), v, 1.0)
    assert np.allclose(out, v.mean(0)) and lse == pytest.approx(math.log(4)) and np.allclose(mag, out)
    out, lse, _, smax = co.attention(np.array([1.0, 0, 0]), np.array([[0.0, 0, 0], [math.log(3), 0, 0]]), v[:2], 1.0)
    assert np.allclose(out, 0.25 * v[0] + 0.75 * v[1]) and smax == pytest.approx(math.log(3))
    assert np.array_equal(co.attention(np.ones(3), np.ones((0, 3)), np.ones((0, 3)), 1.0)[0], np.zeros(3))


# ------------------------------------------------------------------ rotation frequencies
@pytest.mark.parametrize("rot,base,scaling,factor,low,high,context", [
    (128, 10000.0, "none", 1.0, 1.0, 4.0, 8192), (2, 10000.0, "none", 1.0, 1.0, 4.0, 8192),
    (64, 500000.0, "linear", 8.0, 1.0, 4.0, 8192), (128, 10000.0, "base", 4.0, 1.0, 4.0, 8192),
    (128, 500000.0, "bands", 8.0, 1.0, 4.0, 8192), (48, 10000.0, "bands", 3.5, 0.5, 32.0, 4096),
    (128, 10000.0, "ramp", 16.0, 1.0, 32.0, 4096), (256, 1e6, "ramp", 1.0, 1.0, 32.0, 32768),
    (16, 10000.0, "ramp", 4.0, 1.0, 1.001, 1000)])
def test_rope_freqs_match_the_formulas(vla, rot, base, scaling, factor, low, high, context):
    f, scale = vla.rope_freqs(rot, base, scaling, factor, low, high, context, device="cpu")
    ref, ref_scale = co.rope_freqs(rot, base, scaling, factor, low, high, context)
    # a power moves by log(base) <= 14 times its exponent's rounding, 14 * 2^-53 = 1.6e-15, a few times over
    assert np.allclose(f.numpy(), ref, rtol=1e-13, atol=0) and scale == pytest.approx(ref_scale, rel=2.0 ** -23)


def test_rope_scalings_meet_their_ends(vla):
    plain = vla.rope_freqs(128, device="cpu")[0].numpy()
    base = vla.rope_freqs(128, scaling="base", factor=4.0, device="cpu")[0].numpy()
    assert base[0] == plain[0] and base[-1] == pytest.approx(plain[-1] / 4, rel=1e-12)
    bands = vla.rope_freqs(128, scaling="bands", factor=8.0, device="cpu")[0].numpy()
    turns = 8192 * plain / (2 * math.pi)
    assert np.array_equal(bands[turns >= 4], plain[turns >= 4])
    assert np.allclose(bands[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15)
    for s in ("linear", "base", "bands", "ramp"):
        f, scale = vla.rope_freqs(128, scaling=s, factor=1.0, high=32.0, device="cpu")
        assert np.allclose(f.numpy(), plain, rtol=1e-14) and scale == 1.0


@pytest.mark.parametrize("args", [(0, 1e4, 0, 1, 1, 4, 8192), (3, 1e4, 0, 1, 1, 4, 8192), (258, 1e4, 0, 1, 1, 4, 8192),
                                  (64, 1.0, 0, 1, 1, 4, 8192), (64, math.nan, 0, 1, 1, 4, 8192), (64, 1e4, 5, 1, 1, 4, 8192),
                                  (64, 1e4, -1, 1, 1, 4, 8192), (64, 1e4, 1, 0.5, 1, 4, 8192),
                                  (64, 1e4, 1, math.inf, 1, 4, 8192), (2, 1e4, 2, 2, 1, 4, 8192), (64, 1e4, 3, 2, 4, 4, 8192),
                                  (64, 1e4, 3, 2, 0, 4, 8192), (64, 1e4, 4, 2, 1, 4, 0)])
def test_rope_freqs_refusals(vla, args):
    buf = (ctypes.c_double * 256)()
    assert vla.load_library().vla_rope_freqs(*args, buf, None) == -1
    assert vla.load_library().vla_last_error()


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


def test_plan_refusals(vla):
    good = dict(n_env=4, cached=P, new=2 * P, table=P, ld=8, max_pages=8, free=P, n_free=4, head=P, n_pages=64, max_rows=8,
                lens=3 * P, start=P, pos=P, env=P, slot=P, stats=2 * P, stream=None)
    _each(vla, "vla_kv_plan", good, [
        (-1, dict(n_env=-1)), (-1, dict(max_pages=-1)), (-1, dict(n_free=-1)), (-1, dict(n_pages=-1)), (-1, dict(max_rows=-1)),
        (-7, dict(n_pages=1 << 27)), (-7, dict(max_pages=1 << 27, ld=1 << 27)), (-1, dict(ld=7)), (-1, dict(cached=None)),
        (-1, dict(new=None)), (-1, dict(table=None)), (-1, dict(free=None)), (-1, dict(lens=None)), (-1, dict(start=None)),
        (-1, dict(pos=None)), (-1, dict(env=None)), (-1, dict(slot=None)), (-1, dict(stats=None)), (-1, dict(lens=P)),
        (-1, dict(lens=2 * P)), (-1, dict(stats=P))])


def test_norm_rope_refusals(vla):
    good = dict(rows=4, heads=8, kv=2, hd=128, dtype=0, q=P, ld_q=1024, k=P, ld_k=256, v=P, ld_v=256, qg=P, kg=P, eps=1e-6,
                pos=P, freqs=P, rot=128, layout=0, scale=1.0, qo=2 * P, ld_qo=1024, ko=2 * P, ld_ko=256, kp=P, vp=P,
                n_pages=4, slot=P, stream=None)
    _each(vla, "vla_qk_norm_rope", good, [
        (-1, dict(rows=-1)), (-1, dict(heads=0)), (-1, dict(kv=0)), (-7, dict(heads=1 << 16)), (-7, dict(hd=96)),
        (-7, dict(dtype=2)), (-7, dict(rot=24)), (-7, dict(rot=144)), (-7, dict(rot=-16)), (-1, dict(layout=2)),
        (-1, dict(eps=-1.0)), (-1, dict(eps=math.nan)), (-1, dict(scale=math.inf)), (-1, dict(pos=None)),
        (-1, dict(freqs=None)), (-1, dict(freqs=P + 8)), (-1, dict(v=None)), (-1, dict(kp=None)), (-1, dict(vp=None)),
        (-1, dict(slot=None)), (-1, dict(v=None, kp=None, vp=None, slot=None, ko=None)), (-1, dict(q=None)),
        (-1, dict(k=None)), (-1, dict(qo=None)), (-1, dict(q=P + 2)), (-1, dict(ld_q=1016)), (-1, dict(ld_q=1028)),
        (-1, dict(ld_k=0)), (-1, dict(ld_qo=8)), (-1, dict(ko=P + 8)), (-1, dict(ld_v=8)), (-1, dict(qo=P, ld_qo=2048)),
        (-1, dict(ko=P, ld_ko=512)), (-1, dict(qg=P + 4)), (-1, dict(kp=P + 4)), (-1, dict(n_pages=-1)),
        (-7, dict(n_pages=1 << 27))])
    assert _call(vla, "vla_qk_norm_rope", good, rows=0, q=None, k=None)[0] == 0


def test_norm_rope_backward_refusals(vla):
    good = dict(rows=4, heads=8, kv=2, hd=64, dtype=1, q=P, ld_q=512, k=P, ld_k=128, dqo=P, ld_dqo=512, dko=P, ld_dko=128,
                qg=P, kg=P, eps=1e-6, pos=P, freqs=P, rot=64, layout=1, scale=1.0, dq=2 * P, ld_dq=512, dk=2 * P, ld_dk=128,
                dqg=P, dkg=P, ws=P, bytes=1 << 30, stream=None)
    _each(vla, "vla_qk_norm_rope_backward", good, [
        (-1, dict(rows=-1)), (-7, dict(hd=32)), (-7, dict(dtype=-1)), (-1, dict(dqg=None)), (-1, dict(dkg=None)),
        (-3, dict(ws=None)), (-3, dict(bytes=1024)), (-3, dict(ws=P + 4)), (-7, dict(rot=8)), (-1, dict(q=None)),
        (-1, dict(k=None)), (-1, dict(dqo=None)), (-1, dict(dko=None)), (-1, dict(dq=None)), (-1, dict(dk=None)),
        (-1, dict(ld_dk=64)), (-1, dict(dq=P, ld_dq=1024)), (-1, dict(dk=P, ld_dk=256)), (-1, dict(pos=None))])
    none = dict(rows=0, qg=None, kg=None, ws=None, bytes=0, q=None)
    assert _call(vla, "vla_qk_norm_rope_backward", good, **none)[0] == 0
    n = ctypes.c_size_t()
    assert vla.load_library().vla_qk_norm_rope_workspace_size(128, ctypes.byref(n)) == 0 and n.value > 0
    assert vla.load_library().vla_qk_norm_rope_workspace_size(100, ctypes.byref(n)) == -7
    assert vla.load_library().vla_qk_norm_rope_workspace_size(128, None) == -1


def test_attention_refusals(vla):
    good = dict(n_env=4, heads=8, kv=2, hd=128, dtype=0, q=P, ld_q=1024, kp=P, vp=P, n_pages=9, table=P, ld=8, max_pages=8,
                lens=P, scale=0.1, out=2 * P, ld_o=1024, lse=None, ws=P, bytes=1 << 40, stream=None)
    _each(vla, "vla_paged_attention", good, [
        (-1, dict(n_env=-1)), (-7, dict(n_env=1 << 16)), (-1, dict(max_pages=-1)), (-7, dict(max_pages=1 << 26, ld=1 << 26)),
        (-1, dict(kv=3)), (-1, dict(kv=0)), (-7, dict(hd=80)), (-7, dict(dtype=7)), (-1, dict(n_pages=-1)),
        (-7, dict(n_pages=1 << 27)), (-1, dict(scale=math.nan)), (-1, dict(q=None)), (-1, dict(out=None)), (-1, dict(ld_q=8)),
        (-1, dict(ld_o=1000)), (-1, dict(ld=7)), (-1, dict(table=None)), (-1, dict(lens=None)), (-1, dict(kp=None)),
        (-1, dict(vp=None)), (-1, dict(kp=P + 8)), (-3, dict(ws=None)), (-3, dict(bytes=0)), (-3, dict(ws=P + 16))])
    assert _call(vla, "vla_paged_attention", good, n_env=0, q=None, out=None, ws=None)[0] == 0
    n = ctypes.c_size_t()
    lib = vla.load_library()
    assert lib.vla_paged_attention_workspace_size(4, 8, 2, 128, 8, ctypes.byref(n)) == 0
    assert lib.vla_paged_attention_workspace_size(4, 8, 3, 128, 8, ctypes.byref(n)) == -1
    assert lib.vla_paged_attention_workspace_size(4, 8, 2, 128, 8, None) == -1


def test_binding_refuses_host_tensors(vla):
    import torch
    t = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: vla.qk_norm_rope(t, t, i, torch.ones(32, dtype=torch.float64)),
                 lambda: vla.qk_norm_rope_backward(t, t, t, t, i, torch.ones(32, dtype=torch.float64)),
                 lambda: vla.paged_attention(t, t[None], t[None], i[:, None], i, 0.1),
                 lambda: vla.kv_plan(i, i, i[:, None], i, 2, 4)):
        with pytest.raises(ValueError):
            call()
