"""psa_rotary's host side: the spectrum that it fills in, and what it refuses before any launch."""
import ctypes
import math

import pytest

import paper_2512_04025_amd as psa


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(psa.library_path()):
        from paper_2512_04025_amd.build import build_library
        build_library(verbose=False)
    return psa.load_library()


@pytest.mark.parametrize("d,pairs,shared", [(128, (22, 21, 21), False), (128, (16, 24, 24), True), (64, (12, 10, 10), False), (64, (7, 5), False), (64, (0, 32), False), (128, (64,), True)])
def test_spectrum(lib, d, pairs, shared):
    r = psa.make_rotary(d, pairs, base=5000.0, shared=shared)
    assert r.axes == len(pairs)
    i = 0
    for a, n in enumerate(pairs):
        for j in range(n):
            assert r.axis[i] == a
            assert r.freq[i] == pytest.approx(5000.0 ** (-i / (d // 2) if shared else -j / n), rel=1e-14)
            i += 1
    assert all(r.axis[x] == psa.PSA_ROTARY_STILL and r.freq[x] == 0.0 for x in range(i, 64))


@pytest.mark.parametrize("d,pairs,base", [(96, (8, 8), 1e4), (64, (), 1e4), (64, (1,) * 5, 1e4), (64, (20, 20), 1e4), (64, (-1, 8), 1e4), (64, (8, 8), 0.5),
                                          (64, (8, 8), math.inf), (64, (8, 8), math.nan), (64, (2**31 - 1, 2**31 - 1), 1e4)])
def test_spectrum_refuses(lib, d, pairs, base):
    with pytest.raises(psa.PsaError) as e:
        psa.make_rotary(d, pairs, base=base)
    assert e.value.status == 1


def _call(lib, p, r, pos=256, stride=0, perm=None, inverse=0, q=(512, 1024), k=(2048, 4096)):
    v = ctypes.c_void_p
    return lib.psa_rotary(ctypes.byref(p), ctypes.byref(r) if r else None, v(pos), stride, v(perm), inverse, v(q[0]), v(k[0]), v(q[1]), v(k[1]), None)


def test_refusals_before_any_launch(lib):
    """The pointers are never dereferenced: every call fails in validation."""
    p = psa.make_params(2, 4, 2, 100, 64, 64, 64, 4)
    ok = lambda **kw: psa.make_rotary(64, (12, 10, 10), **kw)                       # noqa: E731
    assert _call(lib, p, None) == 1
    assert _call(lib, p, ok(), pos=None) == 1
    assert _call(lib, p, ok(), stride=-1) == 1
    assert _call(lib, p, ok(), q=(512, None)) == 1
    assert _call(lib, p, ok(), k=(None, 512)) == 1
    assert _call(lib, p, ok(), q=(None, None), k=(None, None)) == 1
    assert _call(lib, p, ok(pairing=2)) == 1
    assert _call(lib, p, ok(), q=(512, 512), perm=256) == 1                          # in place and permuted
    assert _call(lib, p, ok(q=(25600, 64, 256)), q=(512, 512)) == 1                  # in place from another layout
    for q, k in (((512, 2048), (2048, 4096)), ((512, 4096), (2048, 4096)), ((512, 1024), (2048, 512))):      # one tensor's output at the other's address
        assert _call(lib, p, ok(), q=q, k=k) == 1
    for bad in (0, 5):
        r = ok()
        r.axes = bad
        assert _call(lib, p, r) == 1
    r = ok()
    r.axis[3] = 3
    assert _call(lib, p, r) == 1
    for f in (math.nan, math.inf, -math.inf, 2.0 ** 20 + 1):
        r = ok()
        r.freq[0] = f
        assert _call(lib, p, r) == 1
    assert _call(lib, p, ok(q=(-1, 64, 256))) == 1
    assert _call(lib, p, ok(q=(2**62, 64, 256))) == 1
    # rows that an inverse call would write twice
    for q in ((0, 6400, 64), (25600, 0, 64), (25600, 6400, 32), (25600, 64, 255), (25536, 64, 256), (6400, 6400, 64)):
        assert _call(lib, p, ok(q=q), inverse=1) == 1, q
    big = psa.make_params(600, 60, 60, 32768, 64, 64, 64, 4)
    assert _call(lib, big, ok()) == 2
    assert _call(lib, psa.make_params(2, 4, 3, 100, 64, 64, 64, 4), ok()) == 1
