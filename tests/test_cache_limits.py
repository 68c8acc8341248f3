"""Limits of the paged cache's operators (vla_cache.h): calls that are refused before any device work."""
import ctypes
import os

import pytest

P = 1 << 20  # an aligned address that is never read: the checks fail first


@pytest.fixture(scope="module")
def lib():
    from paper_2505_18719_amd import vla as binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2505_18719_amd import build
        build.build(verbose=False)
    return binding.load_library()


def ceil(a, b):
    return -(-a // b)


def first_refused(kv, hd, cache):
    """The least number of rows whose launch has 2^24 workgroups of 256 threads or more."""
    lo, hi = 1 << 12, 1 << 27
    while lo < hi:
        r = (lo + hi) // 2
        if ceil(r, 4) + (ceil(r, 16) * ceil(kv * hd, 256) if cache else 0) >= 1 << 24:
            hi = r
        else:
            lo = r + 1
    return lo


@pytest.mark.parametrize("kv,hd,cache", [(1, 64, False), (1, 64, True), (8, 128, True), (1024, 256, True)])
def test_norm_rope_refuses_more_rows_than_a_launch_takes(lib, kv, hd, cache):
    least = first_refused(kv, hd, cache)
    if not cache:
        assert least == 2 ** 26 - 3
    w = kv * hd
    for rows in (least, least + 1, 2 ** 28, 2 ** 31 - 1):
        c = (P, w, P, P, 4, P) if cache else (None, 0, None, None, 0, None)
        rc = lib.vla_qk_norm_rope(rows, kv, kv, hd, 0, P, w, P, w, c[0], c[1], None, None, 1e-6, P, P, 64, 0, 1.0, 2 * P, w,
                                  2 * P, w, c[2], c[3], c[4], c[5], None)
        assert rc == -7 and b"rows" in lib.vla_last_error(), (rows, rc)


@pytest.mark.parametrize("scale", [2.4e38, -3.4e38])
def test_attention_refuses_a_scale_without_room_for_base_2(lib, scale):
    rc = lib.vla_paged_attention(4, 8, 2, 128, 0, P, 1024, P, P, 9, P, 8, 8, P, scale, 2 * P, 1024, None, P, 1 << 40, None)
    assert rc == -1 and b"scale" in lib.vla_last_error()


@pytest.mark.parametrize("rot,base,factor", [(64, 1e300, 1e9), (4, 1e4, 1e160)])
def test_rope_freqs_refuses_a_changed_base_past_64_bits(lib, rot, base, factor):
    buf = (ctypes.c_double * 256)()
    assert lib.vla_rope_freqs(rot, base, 2, factor, 1.0, 4.0, 8192.0, buf, None) == -1 and b"base" in lib.vla_last_error()
