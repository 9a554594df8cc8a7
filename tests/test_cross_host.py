"""The cross attention's host side: workspace sizes, what is refused before any launch, and the 64-bit oracle against differences."""
import ctypes
import os

import numpy as np
import pytest

import paper_2512_04025_amd as psa
from tests import cross_oracle


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(psa.library_path()):
        from paper_2512_04025_amd.build import build_library
        build_library(verbose=False)
    return psa.load_library()


def _fwd(lib, p, x, Q=256, K=512, V=768, O=1024, scratch=256):
    v = ctypes.c_void_p
    return lib.psa_cross_attention_fwd(ctypes.byref(p), ctypes.byref(x) if x else None, v(Q), v(K), v(V), None, None, v(O), None, v(scratch), None)


def _bwd(lib, p, x, **kw):
    a = dict(Q=256, K=512, V=768, O=1024, lse=1280, dO=1536, dQ=1792, dK=2048, dV=2304, scratch=2560)
    a.update(kw)
    v = ctypes.c_void_p
    return lib.psa_cross_attention_bwd(ctypes.byref(p), ctypes.byref(x) if x else None, v(a["Q"]), v(a["K"]), v(a["V"]), None, None, v(a["O"]), v(a["lse"]), v(a["dO"]),
                                       v(a["dQ"]), v(a["dK"]), v(a["dV"]), v(a["scratch"]), None)


def test_refusals_before_any_launch(lib):
    """The pointers are never dereferenced: every call fails in validation."""
    p = psa.make_params(2, 4, 2, 100, 64, 64, 64, 4)
    x = psa.make_cross
    assert _fwd(lib, p, None) == 1 and _bwd(lib, p, None) == 1
    for miss in ("Q", "K", "V", "O"):
        assert _fwd(lib, p, x(50), **{miss: None}) == 1
    for miss in ("Q", "K", "V", "O", "lse", "dO", "dQ", "dK", "dV", "scratch"):
        assert _bwd(lib, p, x(50), **{miss: None}) == 1
    assert _fwd(lib, p, x(-1)) == 1 and _bwd(lib, p, x(-1)) == 1
    causal = psa.make_params(2, 4, 2, 100, 64, 64, 64, 4, causal=True)
    assert _fwd(lib, causal, x(50)) == 1 and _bwd(lib, causal, x(50)) == 1
    assert _bwd(lib, p, x(50), scratch=2560 + 16) == 1
    one = psa.make_params(1, 1, 1, 1, 64, 64, 64, 4)
    assert psa.psa_query_cross_sizes(one, 30000)[0] > 0
    assert _fwd(lib, one, x(30000), scratch=None) == 1 and _fwd(lib, one, x(30000), scratch=264) == 1
    for name in ("q", "k", "v", "o"):
        assert _fwd(lib, p, x(50, **{name: (-64, 64, 64)})) == 1
        assert _fwd(lib, p, x(50, **{name: (2**60, 64, 64)})) == 1
    assert _fwd(lib, p, x(50, o=(0, 6400, 64))) == 1 and _fwd(lib, p, x(50, o=(25600, 0, 64))) == 1 and _fwd(lib, p, x(50, o=(25600, 64, 32))) == 1
    for name in ("dq", "dk", "dv"):
        assert _bwd(lib, p, x(50, **{name: (0, 6400, 64)})) == 1
    # from one token or state to the next at most 32 MB
    for name in ("q", "k", "v", "o"):
        assert _fwd(lib, p, x(50, **{name: (2**40, 2**33, 2**24)})) == 2
    for name in ("q", "k", "v", "o", "do", "dq", "dk", "dv"):
        assert _bwd(lib, p, x(50, **{name: (2**40, 2**33, 2**24)})) == 2
    wide = psa.make_params(1100, 60, 60, 4, 64, 64, 64, 4)
    assert _fwd(lib, wide, x(50)) == 2
    long_ = psa.make_params(1, 1024, 1, 4000000, 64, 64, 64, 4)
    assert _fwd(lib, long_, x(50)) == 2
    assert _fwd(lib, p, x(2**31 - 100)) == 2
    with pytest.raises(psa.PsaError):
        psa.psa_query_cross_sizes(p, -1)


def test_outputs_at_another_tensors_address_are_refused(lib):
    p = psa.make_params(2, 4, 2, 100, 64, 64, 64, 4)
    x = psa.make_cross(50)
    for other in ("Q", "K", "V"):
        assert _fwd(lib, p, x, **{other: 1024}) == 1, other
    at = dict(Q=256, K=512, V=768, O=1024, dO=1536, dQ=1792, dK=2048, dV=2304)
    for out in ("dQ", "dK", "dV"):
        for other in at:
            if other != out:
                assert _bwd(lib, p, x, **{out: at[other]}) == 1, (out, other)


@pytest.mark.parametrize("B,Hq,Hkv,N,M,d", [(1, 12, 12, 32760, 512, 128), (1, 40, 40, 75600, 512, 128), (2, 4, 2, 100, 0, 64), (8, 28, 4, 1, 77, 128), (1, 1, 1, 1, 30000, 64), (2, 16, 16, 64, 32760, 64)])
def test_sizes(lib, B, Hq, Hkv, N, M, d):
    p = psa.make_params(B, Hq, Hkv, N, d, 128, 64, 4)
    fwd, bwd = psa.psa_query_cross_sizes(p, M)
    assert fwd % 256 == 0 and bwd % 256 == 0
    assert bwd >= 4 * B * Hq * N                                                    # a sum per query row
    rows = -(-Hq // Hkv * N // 128) * B * Hkv
    if rows >= 512 or M <= 256:
        assert fwd == 0                                                             # enough blocks of rows for the chip, or nothing to share
    elif M >= 4096:
        assert fwd >= 2 * 4 * B * Hq * N * (d + 1)


@pytest.mark.parametrize("B,Hq,Hkv,N,M,d", [(8, 28, 4, 1, 1500, 128), (2, 8, 2, 40, 3000, 64), (1, 28, 4, 33, 65, 128)])
def test_sizes_do_not_depend_on_strides(lib, B, Hq, Hkv, N, M, d):
    """Heads of a group may be one run of rows or not: the workspace is enough for both."""
    for dtype in (psa.PSA_BF16, psa.PSA_F32):
        p = psa.make_params(B, Hq, Hkv, N, d, 128, 64, 4, dtype=dtype)
        tokens = (N * Hq * d, d, Hq * d)
        assert psa.psa_query_cross_sizes(p, M) == psa.psa_query_cross_sizes(p, psa.make_cross(M, q=tokens, o=tokens, dq=tokens, do=tokens))


def test_oracle_gradients_are_differences():
    rng = np.random.default_rng(5)
    Q, dO = rng.standard_normal((1, 4, 3, 8)), rng.standard_normal((1, 4, 3, 8))
    K, V = rng.standard_normal((1, 2, 5, 8)), rng.standard_normal((1, 2, 5, 8))
    vis = np.array([[True, False, True, True, True]])
    f = lambda: (cross_oracle.forward(Q, K, V, vis, 0.4, "f32")[0] * dO).sum()      # noqa: E731
    O, lse, _, _ = cross_oracle.forward(Q, K, V, vis, 0.4, "f32")
    grads, _ = cross_oracle.backward(Q, K, V, O, lse, dO, vis, 0.4, "f32")
    for x, g in zip((Q, K, V), grads):
        for at in [tuple(rng.integers(0, n) for n in x.shape) for _ in range(12)]:
            keep, h = x[at], 1e-5
            x[at] = keep + h
            up = f()
            x[at] = keep - h
            down = f()
            x[at] = keep
            assert (up - down) / (2 * h) == pytest.approx(g[at], rel=1e-6, abs=1e-8)
