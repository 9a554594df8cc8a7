"""ctypes binding of libpsa.so: same entry-point names as include/psa.h, argument marshalling only."""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence, Tuple

PSA_OK, PSA_EINVAL, PSA_EUNSUPPORTED, PSA_ELAUNCH = 0, 1, 2, 3
PSA_BF16, PSA_F32 = 0, 1
PSA_REP_STRIDED, PSA_REP_POOLED = 0, 1
PSA_EST_MAX, PSA_EST_MEAN = 0, 1
PSA_ALLOC_THRESHOLD, PSA_ALLOC_QUANTILE, PSA_ALLOC_BUDGET, PSA_ALLOC_THRESHOLD_EXCL = 0, 1, 2, 3
PSA_CAP_PER_HEAD, PSA_CAP_ALL_HEADS = 0, 1
PSA_ROTARY_ADJACENT, PSA_ROTARY_HALVES = 0, 1
PSA_ROTARY_MAX_AXES, PSA_ROTARY_STILL = 4, 255
PSA_MAX_LEVELS = 8

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libpsa.so")
_lib = None


class PsaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {psa_status_str(status)} (status {status})")


class PsaParams(ctypes.Structure):
    """Mirror of `psa_params` in include/psa.h."""
    _fields_ = [
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("N", ctypes.c_int32),
        ("d", ctypes.c_int32), ("bq", ctypes.c_int32), ("bk", ctypes.c_int32), ("levels", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("scale", ctypes.c_float),
        ("sq", ctypes.c_int32), ("sk", ctypes.c_int32), ("rep_mode", ctypes.c_int32),
        ("est_pool", ctypes.c_int32), ("alloc_mode", ctypes.c_int32),
        ("tau", ctypes.c_float * PSA_MAX_LEVELS), ("budget", ctypes.c_float),
    ]

    @property
    def nq(self) -> int:
        return -(-self.N // self.bq)

    @property
    def nk(self) -> int:
        return -(-self.N // self.bk)


def _stride_field(name: str):
    """A spec's strides as a tuple: kept beside the struct's words, since every call compares them with its tensors."""
    words, kept = "_" + name, "_" + name + "_tuple"

    def get(self):
        return getattr(self, kept, (0, 0, 0))

    def put(self, strides):
        b, h, n = (int(s) for s in strides)
        setattr(self, words, (b, h, n))
        setattr(self, kept, (b, h, n))
    return property(get, put)


class PsaRotary(ctypes.Structure):
    """Mirror of `psa_rotary_spec` in include/psa.h (see make_rotary)."""
    _fields_ = [
        ("axes", ctypes.c_int32), ("pairing", ctypes.c_int32), ("axis", ctypes.c_uint8 * 64), ("freq", ctypes.c_double * 64),
        ("_q_stride", ctypes.c_int64 * 3), ("_k_stride", ctypes.c_int64 * 3),
    ]
    q_stride, k_stride = _stride_field("q_stride"), _stride_field("k_stride")


class PsaCross(ctypes.Structure):
    """Mirror of `psa_cross` in include/psa.h (see make_cross)."""
    _fields_ = [("M", ctypes.c_int32)] + [("_" + n + "_stride", ctypes.c_int64 * 3) for n in ("q", "k", "v", "o", "dq", "dk", "dv", "do")]
    q_stride, k_stride, v_stride, o_stride = (_stride_field(n + "_stride") for n in "qkvo")
    dq_stride, dk_stride, dv_stride, do_stride = (_stride_field("d" + n + "_stride") for n in "qkvo")


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load libpsa.so built in-tree.  There is no fallback: without the HIP library nothing runs."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2512_04025_amd.build` "
            "(hipcc, gfx950).  There is no CPU or PyTorch fallback.")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, pp = ctypes.c_void_p, ctypes.POINTER(PsaParams)
    szp = ctypes.POINTER(ctypes.c_size_t)
    lib.psa_query_sizes.argtypes = [pp, szp, szp]
    lib.psa_build_pyramid.argtypes = [pp, vp, vp, vp, vp, vp]
    fp = ctypes.POINTER(ctypes.c_float)
    lib.psa_hilbert_order.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]
    lib.psa_permute_tokens.argtypes = [pp, ctypes.c_int32, vp, vp, ctypes.c_int32, vp, vp]
    rp = ctypes.POINTER(PsaRotary)
    lib.psa_rotary_spectrum.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), ctypes.c_double, ctypes.c_int32, rp]
    lib.psa_rotary.argtypes = [pp, rp, vp, ctypes.c_int64, vp, ctypes.c_int32, vp, vp, vp, vp, vp]
    xp = ctypes.POINTER(PsaCross)
    lib.psa_query_cross_sizes.argtypes = [pp, xp, szp, szp]
    lib.psa_cross_attention_fwd.argtypes = [pp, xp] + [vp] * 9
    lib.psa_cross_attention_bwd.argtypes = [pp, xp] + [vp] * 13
    lib.psa_level_cap.argtypes = [pp, vp, fp, ctypes.c_int, vp, vp, vp]
    lib.psa_build_pyramid_cap.argtypes = [pp, vp, vp, vp, vp, fp, ctypes.c_int, vp, vp, vp]
    lib.psa_allocate_levels.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.psa_attention_fwd.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.psa_attention_fwd_static.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.psa_query_bwd_sizes.argtypes = [pp, szp]
    lib.psa_attention_bwd.argtypes = [pp] + [vp] * 14
    lib.psa_dense_ref.argtypes = [pp, vp, vp, vp, vp, vp, vp]
    lib.psa_probe_copy.argtypes = [vp, vp, ctypes.c_size_t, vp]
    lib.psa_probe_mfma.argtypes = [vp, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_double), vp]
    lib.psa_status_str.argtypes = [ctypes.c_int]
    lib.psa_status_str.restype = ctypes.c_char_p
    for name in ("psa_query_sizes", "psa_build_pyramid", "psa_allocate_levels", "psa_attention_fwd", "psa_attention_fwd_static",
                 "psa_level_cap", "psa_build_pyramid_cap", "psa_query_bwd_sizes", "psa_attention_bwd", "psa_hilbert_order", "psa_permute_tokens",
                 "psa_dense_ref", "psa_probe_copy", "psa_probe_mfma", "psa_rotary_spectrum", "psa_rotary",
                 "psa_query_cross_sizes", "psa_cross_attention_fwd", "psa_cross_attention_bwd"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def make_params(B: int, Hq: int, Hkv: int, N: int, d: int, bq: int, bk: int, levels: int,
                dtype: int = PSA_BF16, causal: bool = False, scale: float = 0.0, sq: int = 0, sk: int = 0,
                rep_mode: int = PSA_REP_POOLED, est_pool: int = PSA_EST_MAX,
                alloc_mode: int = PSA_ALLOC_BUDGET, tau: Sequence[float] = (), budget: float = 0.25) -> PsaParams:
    p = PsaParams()
    p.B, p.Hq, p.Hkv, p.N, p.d = B, Hq, Hkv, N, d
    p.bq, p.bk, p.levels = bq, bk, levels
    p.dtype, p.causal, p.scale = dtype, int(bool(causal)), scale
    p.sq, p.sk, p.rep_mode, p.est_pool, p.alloc_mode = sq, sk, rep_mode, est_pool, alloc_mode
    for i, t in enumerate(tau):
        p.tau[i] = t
    p.budget = budget
    return p


def _ptr(t) -> Optional[int]:
    """Device pointer of a torch tensor (None stays NULL).  Tensors must be contiguous CUDA tensors."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("libpsa takes contiguous device tensors")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream or None
    return getattr(stream, "cuda_stream", stream) or None


def _check(status: int, where: str) -> None:
    if status != PSA_OK:
        raise PsaError(status, where)


def psa_status_str(status: int) -> str:
    return load_library().psa_status_str(status).decode()


def psa_query_sizes(p: PsaParams) -> Tuple[int, int]:
    """(bytes of one pyramid buffer, bytes of scratch)."""
    pyr, scr = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(load_library().psa_query_sizes(ctypes.byref(p), ctypes.byref(pyr), ctypes.byref(scr)), "psa_query_sizes")
    return pyr.value, scr.value


def psa_build_pyramid(p: PsaParams, K, V, Kpyr, Vpyr, stream=None) -> None:
    _check(load_library().psa_build_pyramid(ctypes.byref(p), _ptr(K), _ptr(V), _ptr(Kpyr), _ptr(Vpyr),
                                            _stream(stream)), "psa_build_pyramid")


def psa_hilbert_order(T: int, Hg: int, W: int):
    """Host call: the Hilbert-curve token order of a T x Hg x W grid as a numpy int32 array."""
    import numpy as np
    perm = np.empty(T * Hg * W, dtype=np.int32)
    _check(load_library().psa_hilbert_order(T, Hg, W, perm.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))),
           "psa_hilbert_order")
    return perm


def psa_permute_tokens(p: PsaParams, X, perm, Y, inverse: bool = False, stream=None) -> None:
    """X, Y: [..., N, d] device tensors of p's dtype (all leading axes are heads); perm: device int32 [N]."""
    heads = X.numel() // (p.N * p.d)
    _check(load_library().psa_permute_tokens(ctypes.byref(p), ctypes.c_int32(heads), _ptr(X), _ptr(perm),
                                             ctypes.c_int32(1 if inverse else 0), _ptr(Y), _stream(stream)),
           "psa_permute_tokens")


def _strides_of(x) -> Tuple[int, int, int]:
    """Strides (batch, head, token) that a spec gets: of a [B, H, L, d] tensor or view, as a tuple, or None (contiguous)."""
    if x is None:
        return (0, 0, 0)
    if isinstance(x, (tuple, list)):
        b, h, n = x
        return (int(b), int(h), int(n))
    if x.dim() != 4 or x.stride(3) != 1:
        raise ValueError("libpsa takes [B, H, L, d] tensors whose channels are adjacent")
    return (0, 0, 0) if x.is_contiguous() else tuple(x.stride()[:3])


_CONTIGUOUS = (0, 0, 0)


def _rows(x, shape, dtype, strides, device: int):
    """Device pointer of a [B, H, L, d] tensor that the kernels address by `strides` ((0, 0, 0): contiguous)."""
    if x is None:
        return None
    if x.shape != shape or x.dtype is not dtype or x.get_device() != device:
        raise ValueError(f"expected a {dtype} tensor of shape {tuple(shape)} on the current device, got {x.dtype} {tuple(x.shape)} on {x.device}")
    if strides == _CONTIGUOUS:
        if not x.is_contiguous():
            raise ValueError("the tensor is not contiguous: give its strides to the spec")
    elif x.stride() != strides + (1,) and x.numel():
        for n, want, got in zip(shape, strides + (1,), x.stride()):
            if n > 1 and want != got:
                raise ValueError(f"the tensor's strides {x.stride()} are not the spec's {strides}")
    return x.data_ptr()


def _table(x, shapes, dtype, device: int, what):
    """Device pointer of a contiguous table (None stays NULL)."""
    if x is None:
        return None
    if x.dtype != dtype or x.shape not in shapes or x.get_device() != device or not x.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of shape {' or '.join(map(str, shapes))} on the current device")
    return x.data_ptr()


_torch = None


def _here(p: PsaParams, stream):
    """The library, torch, the current device, its stream to work on, p's element type."""
    global _torch
    torch = _torch
    if torch is None:
        import torch
        torch.cuda.init()
        _torch = torch
    dev = torch._C._cuda_getDevice()
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(dev)
    else:
        stream = getattr(stream, "cuda_stream", stream)
    return _lib or load_library(), torch, dev, stream or None, torch.float32 if p.dtype else torch.bfloat16


def make_rotary(d: int, pairs: Sequence[int], base: float = 10000.0, shared: bool = False, pairing: int = PSA_ROTARY_ADJACENT,
                q=None, k=None) -> PsaRotary:
    """Spec of psa_rotary: `pairs` channel pairs per axis (psa_rotary_spectrum); q, k: the tensors on the tokens' side, or their
    strides (batch, head, token), where those are not contiguous."""
    r = PsaRotary()
    n = (ctypes.c_int32 * max(len(pairs), 1))(*pairs)
    _check(load_library().psa_rotary_spectrum(d, len(pairs), n, base, 1 if shared else 0, ctypes.byref(r)), "psa_rotary_spectrum")
    r.pairing = pairing
    r.q_stride, r.k_stride = _strides_of(q), _strides_of(k)
    return r


def psa_rotary(p: PsaParams, r: PsaRotary, pos, Qin, Kin, Qout, Kout, perm=None, inverse: bool = False, stream=None) -> None:
    """Q and K ([B, heads, N, d], either may be None on both sides) turned by pos (int32 [axes, N], [1, axes, N] or [B, axes, N])."""
    lib, torch, dev, at, dt = _here(p, stream)
    B, N, axes = p.B, p.N, r.axes
    sq, sk = (B, p.Hq, N, p.d), (B, p.Hkv, N, p.d)
    if pos is None:
        raise ValueError("pos is needed")
    loose_q, loose_k, tight = r.q_stride, r.k_stride, _CONTIGUOUS
    if inverse:
        q, k, qo, ko = _rows(Qin, sq, dt, tight, dev), _rows(Kin, sk, dt, tight, dev), _rows(Qout, sq, dt, loose_q, dev), _rows(Kout, sk, dt, loose_k, dev)
    else:
        q, k, qo, ko = _rows(Qin, sq, dt, loose_q, dev), _rows(Kin, sk, dt, loose_k, dev), _rows(Qout, sq, dt, tight, dev), _rows(Kout, sk, dt, tight, dev)
    status = lib.psa_rotary(
        ctypes.byref(p), ctypes.byref(r), _table(pos, ((axes, N), (1, axes, N), (B, axes, N)), torch.int32, dev, "pos"),
        axes * N if pos.dim() == 3 and pos.shape[0] > 1 else 0, _table(perm, ((N,),), torch.int32, dev, "perm"), 1 if inverse else 0, q, k, qo, ko, at)
    if status:
        raise PsaError(status, "psa_rotary")


def _thresholds(p: PsaParams, tau_s: Sequence[float]):
    vals = list(tau_s)
    if len(vals) < p.levels - 1:
        raise ValueError("need levels - 1 similarity thresholds")
    return (ctypes.c_float * max(len(vals), 1))(*vals)


def psa_level_cap(p: PsaParams, K, tau_s: Sequence[float], sim, L, reduce: int = PSA_CAP_PER_HEAD, stream=None) -> None:
    _check(load_library().psa_level_cap(ctypes.byref(p), _ptr(K), _thresholds(p, tau_s), ctypes.c_int(reduce),
                                        _ptr(sim), _ptr(L), _stream(stream)), "psa_level_cap")


def psa_build_pyramid_cap(p: PsaParams, K, V, Kpyr, Vpyr, tau_s: Sequence[float], sim, L,
                          reduce: int = PSA_CAP_PER_HEAD, stream=None) -> None:
    _check(load_library().psa_build_pyramid_cap(ctypes.byref(p), _ptr(K), _ptr(V), _ptr(Kpyr), _ptr(Vpyr),
                                                _thresholds(p, tau_s), ctypes.c_int(reduce), _ptr(sim), _ptr(L),
                                                _stream(stream)), "psa_build_pyramid_cap")


def psa_allocate_levels(p: PsaParams, Q, K, Kpyr, M, scratch, scores_in=None, scores_out=None,
                        level_cap=None, rho_out=None, stream=None) -> None:
    _check(load_library().psa_allocate_levels(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(Kpyr), _ptr(scores_in),
                                              _ptr(scores_out), _ptr(level_cap), _ptr(M), _ptr(rho_out),
                                              _ptr(scratch), _stream(stream)), "psa_allocate_levels")


def psa_attention_fwd(p: PsaParams, Q, K, V, Kpyr, Vpyr, M, O, scratch, lse=None, stream=None) -> None:
    _check(load_library().psa_attention_fwd(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(Kpyr), _ptr(Vpyr),
                                            _ptr(M), _ptr(O), _ptr(lse), _ptr(scratch), _stream(stream)),
           "psa_attention_fwd")


def psa_attention_fwd_static(p: PsaParams, Q, K, V, Kpyr, Vpyr, M, O, lse=None, stream=None) -> None:
    _check(load_library().psa_attention_fwd_static(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(Kpyr),
                                                   _ptr(Vpyr), _ptr(M), _ptr(O), _ptr(lse), _stream(stream)),
           "psa_attention_fwd_static")


def psa_query_bwd_sizes(p: PsaParams) -> int:
    scr = ctypes.c_size_t(0)
    _check(load_library().psa_query_bwd_sizes(ctypes.byref(p), ctypes.byref(scr)), "psa_query_bwd_sizes")
    return scr.value


def psa_attention_bwd(p: PsaParams, Q, K, V, Kpyr, Vpyr, M, O, lse, dO, dQ, dK, dV, scratch, stream=None) -> None:
    _check(load_library().psa_attention_bwd(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(Kpyr), _ptr(Vpyr),
                                            _ptr(M), _ptr(O), _ptr(lse), _ptr(dO), _ptr(dQ), _ptr(dK), _ptr(dV),
                                            _ptr(scratch), _stream(stream)), "psa_attention_bwd")


def psa_dense_ref(p: PsaParams, Q, K, V, O, lse=None, stream=None) -> None:
    _check(load_library().psa_dense_ref(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(lse),
                                        _stream(stream)), "psa_dense_ref")


def make_cross(M: int, q=None, k=None, v=None, o=None, dq=None, dk=None, dv=None, do=None) -> PsaCross:
    """Spec of the cross attention to M states; per tensor the tensor itself ([B, H, L, d], any view with adjacent channels) or its
    strides (batch, head, token) where it is not contiguous."""
    x = PsaCross()
    x.M = M
    for name, t in (("q", q), ("k", k), ("v", v), ("o", o), ("dq", dq), ("dk", dk), ("dv", dv), ("do", do)):
        setattr(x, name + "_stride", _strides_of(t))
    return x


def psa_query_cross_sizes(p: PsaParams, x) -> Tuple[int, int]:
    """(bytes of scratch of the forward call, of the backward call); x: a PsaCross, or just M."""
    fwd, bwd = ctypes.c_size_t(0), ctypes.c_size_t(0)
    x = x if isinstance(x, PsaCross) else make_cross(x)
    _check(load_library().psa_query_cross_sizes(ctypes.byref(p), ctypes.byref(x), ctypes.byref(fwd), ctypes.byref(bwd)), "psa_query_cross_sizes")
    return fwd.value, bwd.value


def _scratch(lib, p: PsaParams, x: PsaCross, scratch, backward: bool, device: int):
    """Device pointer of a workspace that is large enough."""
    need = ctypes.c_size_t(0)
    status = lib.psa_query_cross_sizes(ctypes.byref(p), ctypes.byref(x), None if backward else ctypes.byref(need), ctypes.byref(need) if backward else None)
    if status:
        raise PsaError(status, "psa_query_cross_sizes")
    if scratch is None:
        if need.value:
            raise ValueError(f"{need.value} bytes of scratch are needed")
        return None
    if scratch.get_device() != device or not scratch.is_contiguous() or scratch.numel() * scratch.element_size() < need.value:
        raise ValueError(f"scratch: a contiguous tensor of {need.value} bytes on the current device is needed")
    return scratch.data_ptr()


def _seen(torch, p: PsaParams, x: PsaCross, kv_len, key_mask, device: int):
    """Device pointers of the lengths and the mask."""
    return (_table(kv_len, ((p.B,),), torch.int32, device, "kv_len"),
            None if key_mask is None else _table(key_mask, ((p.B, x.M),), torch.bool if key_mask.dtype == torch.bool else torch.uint8, device, "key_mask"))


def psa_cross_attention_fwd(p: PsaParams, x: PsaCross, Q, K, V, O, scratch=None, lse=None, kv_len=None, key_mask=None, stream=None) -> None:
    """Q, O: [B, Hq, N, d]; K, V: [B, Hkv, M, d]; kv_len: int32 [B]; key_mask: uint8 or bool [B, M]; lse: float [B, Hq, N]."""
    lib, torch, dev, at, dt = _here(p, stream)
    B, Hq, N, d = p.B, p.Hq, p.N, p.d
    sq, sk = (B, Hq, N, d), (B, p.Hkv, x.M, d)
    status = lib.psa_cross_attention_fwd(
        ctypes.byref(p), ctypes.byref(x), _rows(Q, sq, dt, x.q_stride, dev), _rows(K, sk, dt, x.k_stride, dev), _rows(V, sk, dt, x.v_stride, dev),
        *_seen(torch, p, x, kv_len, key_mask, dev), _rows(O, sq, dt, x.o_stride, dev), _table(lse, ((B, Hq, N),), torch.float32, dev, "lse"),
        _scratch(lib, p, x, scratch, False, dev), at)
    if status:
        raise PsaError(status, "psa_cross_attention_fwd")


def psa_cross_attention_bwd(p: PsaParams, x: PsaCross, Q, K, V, O, lse, dO, dQ, dK, dV, scratch, kv_len=None, key_mask=None, stream=None) -> None:
    """O, lse: as the forward call gave them; dO: as O; dQ, dK, dV: as Q, K, V, all written."""
    lib, torch, dev, at, dt = _here(p, stream)
    B, Hq, N, d = p.B, p.Hq, p.N, p.d
    sq, sk = (B, Hq, N, d), (B, p.Hkv, x.M, d)
    status = lib.psa_cross_attention_bwd(
        ctypes.byref(p), ctypes.byref(x), _rows(Q, sq, dt, x.q_stride, dev), _rows(K, sk, dt, x.k_stride, dev), _rows(V, sk, dt, x.v_stride, dev),
        *_seen(torch, p, x, kv_len, key_mask, dev), _rows(O, sq, dt, x.o_stride, dev), _table(lse, ((B, Hq, N),), torch.float32, dev, "lse"),
        _rows(dO, sq, dt, x.do_stride, dev), _rows(dQ, sq, dt, x.dq_stride, dev), _rows(dK, sk, dt, x.dk_stride, dev), _rows(dV, sk, dt, x.dv_stride, dev),
        _scratch(lib, p, x, scratch, True, dev), at)
    if status:
        raise PsaError(status, "psa_cross_attention_bwd")


def psa_probe_copy(src, dst, nbytes: int, stream=None) -> None:
    _check(load_library().psa_probe_copy(_ptr(src), _ptr(dst), ctypes.c_size_t(nbytes), _stream(stream)),
           "psa_probe_copy")


def psa_probe_mfma(sink, workgroups: int, iters: int, random_operands: bool = False, stream=None) -> float:
    """Launches the MFMA-only loop; returns the floating-point operations of the launch."""
    flops = ctypes.c_double(0.0)
    _check(load_library().psa_probe_mfma(_ptr(sink), ctypes.c_int(workgroups), ctypes.c_int(iters),
                                         ctypes.c_int(1 if random_operands else 0), ctypes.byref(flops),
                                         _stream(stream)), "psa_probe_mfma")
    return flops.value
