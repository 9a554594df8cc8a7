"""psa_rotary against its definition in 64 bits: types, pairings, layouts, permutations, far positions, what is left as it was, and the
call beside the ones that it feeds.

Tolerance of a turned pair: sine and cosine are off by at most 2^-22 (the angle's remainder and its product with pi / 2 in 32 bits,
0.79 2^-24 each, Horner's last steps 1.5 2^-24), the two products and the sum round to 2^-24 each: 6 2^-24 (|x0| + |x1|), plus half
a step of the stored type."""
import numpy as np
import pytest

import synth_inputs as si
from tests.psa_testlib import Buffers, gpu_params, oracle_params, to_dev

pytestmark = pytest.mark.gpu

psa = pytest.importorskip("paper_2512_04025_amd")


def oracle(x, pos, spec, d, inverse):
    """x [B, H, N, d], pos [B, axes, N] -> turned rows and |x0| + |x1| of every channel's pair, float64."""
    half = d // 2
    axis, freq = np.array(spec.axis[:half]), np.array(spec.freq[:half])
    still = axis == psa.PSA_ROTARY_STILL
    ang = pos.astype(np.float64)[:, np.where(still, 0, axis)].transpose(0, 2, 1) * freq * (-1.0 if inverse else 1.0)
    c, s = np.where(still, 1.0, np.cos(ang))[:, None], np.where(still, 0.0, np.sin(ang))[:, None]
    a, b = (slice(0, None, 2), slice(1, None, 2)) if spec.pairing == psa.PSA_ROTARY_ADJACENT else (slice(0, half), slice(half, d))
    y, size = np.empty_like(x), np.empty_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size


def limit(y, size, dtype):
    return np.abs(y) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) + 6 * 2.0 ** -24 * size


def torch_dtype(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def rows(shape, dtype, layout, seed, offset=0):
    """[B, H, N, d] on the GPU: contiguous, token by token, or one of three projections side by side, `offset` elements behind an aligned address."""
    import torch
    B, H, N, d = shape
    wide = {"heads": (B, H, N, d), "tokens": (B, N, H, d), "fused": (B, N, 3 * H, d)}[layout]
    g = torch.Generator().manual_seed(seed)
    flat = torch.randn(int(np.prod(wide)) + offset, generator=g).to(torch_dtype(dtype)).cuda()[offset:].view(wide)
    return flat if layout == "heads" else flat[:, :, :H].transpose(1, 2) if layout == "tokens" else flat[:, :, H:2 * H].transpose(1, 2)


def f64(t):
    return t.double().cpu().numpy()


def check(dtype, d, pairing, pairs, shared, B, Hq, Hkv, N, layout, permuted, inverse, per_batch, offset=0, far=3000):
    import torch
    p = psa.make_params(B, Hq, Hkv, N, d, 64, 64, 1, dtype=psa.PSA_BF16 if dtype == "bf16" else psa.PSA_F32)
    rng = np.random.default_rng(N * 7 + d + Hq)
    pos = rng.integers(-far, far, (B if per_batch else 1, len(pairs), N)).astype(np.int32)
    perm = rng.permutation(N).astype(np.int32) if permuted else None
    loose = [rows((B, h, N, d), dtype, layout, 11 + h, offset) for h in (Hq, Hkv)]
    tight = [rows((B, h, N, d), dtype, "heads", 77 + h, offset) for h in (Hq, Hkv)]
    spec = psa.make_rotary(d, pairs, shared=shared, pairing=pairing, q=loose[0], k=loose[1])
    src, dst = (tight, loose) if inverse else (loose, tight)
    given = [f64(x) for x in src]
    psa.psa_rotary(p, spec, torch.from_numpy(pos).cuda(), *src, *dst, perm=None if perm is None else torch.from_numpy(perm).cuda(), inverse=inverse)
    torch.cuda.synchronize()
    posb = np.broadcast_to(pos, (B,) + pos.shape[1:])
    for x, got in zip(given, dst):
        if inverse and perm is not None:
            y = np.empty_like(x)
            y[:, :, perm] = x
            x = y
        want, size = oracle(x, posb, spec, d, inverse)
        if not inverse and perm is not None:
            want, size = want[:, :, perm], size[:, :, perm]
        assert np.all(np.abs(f64(got) - want) <= limit(want, size, dtype))
    return src, dst


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("inverse", [False, True])
def test_types_pairings_layouts(dtype, d, pairing, inverse):
    pairs = {64: (12, 10, 10), 128: (22, 21, 21)}[d]
    for layout, permuted, shared, per_batch in (("heads", False, False, False), ("tokens", True, True, True), ("fused", False, True, False), ("fused", True, False, True)):
        check(dtype, d, pairing, pairs, shared, 2, 6, 3, 117, layout, permuted, inverse, per_batch)


@pytest.mark.parametrize("N", [1, 2, 3, 31, 33, 257, 5003])
def test_lengths(N):
    check("bf16", 128, 0, (22, 21, 21), False, 1, 12, 12, N, "tokens", N % 2 == 1, False, False)
    check("bf16", 128, 1, (16, 24, 24), True, 3, 28, 4, min(N, 700), "heads", False, N % 2 == 1, True)


@pytest.mark.parametrize("B,Hq,Hkv,N", [(1, 1, 1, 40000), (1, 40, 40, 3001), (8, 28, 4, 1), (2, 7, 1, 10001)])
def test_heads_a_thread(B, Hq, Hkv, N):
    """Few and many rows: one head a thread up to eight, runs of heads that do not go into the groups."""
    check("bf16", 64, 1, (12, 10, 10), False, B, Hq, Hkv, N, "tokens", False, False, B > 1)
    check("bf16", 64, 0, (12, 10, 10), False, B, Hq, Hkv, N, "tokens", True, True, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [1, 3])
def test_element_alignment(dtype, offset):
    for inverse in (False, True):
        check(dtype, 64, offset // 2, (12, 10, 10), False, 2, 3, 1, 45, "tokens", False, inverse, False, offset=offset)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_beyond_32_bits(dtype):
    """Tokens 16 MB apart, 270 of them: Q and K end 4.5 GB behind their first element."""
    import torch
    p = psa.make_params(1, 4, 2, 270, 64, 64, 64, 1, dtype=psa.PSA_BF16 if dtype == "bf16" else psa.PSA_F32)
    near = [rows((1, h, 270, 64), dtype, "heads", h) for h in (4, 2)]
    step = 2 ** 24 // near[0].element_size()
    flat = torch.empty(270 * step, dtype=near[0].dtype, device="cuda")
    far = [flat.as_strided(x.shape, (270 * step, 64, step, 1), i * 4 * 64).copy_(x) for i, x in enumerate(near)]
    spec = psa.make_rotary(64, (12, 10, 10), q=far[0], k=far[1])
    pos = torch.arange(3 * 270, dtype=torch.int32, device="cuda").view(3, 270)
    perm = torch.arange(269, -1, -1, dtype=torch.int32, device="cuda")
    out = [torch.empty_like(x) for x in near]
    psa.psa_rotary(p, spec, pos, *far, *out, perm=perm)
    for x, got in zip(near, out):
        want, size = oracle(f64(x), pos[None].cpu().numpy(), spec, 64, False)
        assert np.all(np.abs(f64(got) - want[:, :, ::-1]) <= limit(want, size, dtype)[:, :, ::-1])
    given = [f64(x) for x in out]
    psa.psa_rotary(p, spec, pos, *out, *far, perm=perm, inverse=True)
    for x, got in zip(given, far):
        want, size = oracle(x[:, :, ::-1], pos[None].cpu().numpy(), spec, 64, True)
        assert np.all(np.abs(f64(got) - want) <= limit(want, size, dtype))


@pytest.mark.parametrize("pairing,inverse", [(0, False), (1, True)])
def test_inputs_beyond_the_cache_have_the_bits_of_their_parts(pairing, inverse):
    """276 MB of rows in one call, and a part of the tokens at a time."""
    import torch
    B, H, N, d = 1, 12, 45000, 128
    Q, K = (torch.randn((B, H, N, d), generator=torch.Generator("cuda").manual_seed(i), device="cuda").to(torch.bfloat16) for i in (1, 2))
    pos = torch.randint(-5000, 5000, (3, N), generator=torch.Generator("cuda").manual_seed(3), device="cuda", dtype=torch.int32)
    whole = [torch.empty_like(x) for x in (Q, K)]
    psa.psa_rotary(psa.make_params(B, H, H, N, d, 64, 64, 1), psa.make_rotary(d, (22, 21, 21), pairing=pairing), pos, Q, K, *whole, inverse=inverse)
    for at in (0, 20000, 40000):
        n = min(20000, N - at)
        part = [x[:, :, at:at + n].contiguous() for x in (Q, K)]
        out = [torch.empty_like(x) for x in part]
        psa.psa_rotary(psa.make_params(B, H, H, n, d, 64, 64, 1), psa.make_rotary(d, (22, 21, 21), pairing=pairing), pos[:, at:at + n].contiguous(), *part, *out, inverse=inverse)
        assert all(torch.equal(x[:, :, at:at + n], y) for x, y in zip(whole, out))


def test_far_positions():
    """Angles of 10^7 radians on the fastest channel: the remainder is made in 64 bits (float32 would be off by half a radian)."""
    check("f32", 128, 0, (22, 21, 21), False, 1, 2, 2, 501, "heads", False, False, False, far=10 ** 7)


def test_partial_and_single_axes():
    check("bf16", 128, 1, (10, 7), False, 1, 4, 2, 129, "tokens", False, False, False)
    check("f32", 64, 0, (32,), True, 2, 2, 2, 50, "heads", False, False, True)
    check("f32", 64, 0, (3, 4, 5, 6), False, 1, 2, 2, 50, "heads", True, True, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pairs_that_are_not_turned_keep_their_bits(dtype):
    import torch
    for pairing in (0, 1):
        d, N = 64, 33
        p = psa.make_params(1, 2, 2, N, d, 64, 64, 1, dtype=psa.PSA_BF16 if dtype == "bf16" else psa.PSA_F32)
        spec = psa.make_rotary(d, (5, 6), pairing=pairing)
        x = rows((1, 2, N, d), dtype, "heads", 5)
        still = slice(22, 64) if pairing == 0 else [c for i in range(11, 32) for c in (i, i + 32)]
        special = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0, 0.0], dtype=x.dtype, device="cuda")
        x[..., still] = special[torch.randint(0, 5, x[..., still].shape, generator=torch.Generator().manual_seed(1)).cuda()]
        y = torch.empty_like(x)
        psa.psa_rotary(p, spec, torch.arange(2 * N, dtype=torch.int32, device="cuda").view(2, N), x, None, y, None)
        bits = torch.int16 if dtype == "bf16" else torch.int32
        assert torch.equal(y.view(bits)[..., still], x.view(bits)[..., still])


def test_in_place_one_tensor_and_rows_without_an_index():
    import torch
    N, d = 77, 128
    p = psa.make_params(2, 4, 2, N, d, 64, 64, 1)
    spec = psa.make_rotary(d, (22, 21, 21))
    pos = torch.randint(0, 100, (3, N), dtype=torch.int32).cuda()
    q, k = rows((2, 4, N, d), "bf16", "heads", 1), rows((2, 2, N, d), "bf16", "heads", 2)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    psa.psa_rotary(p, spec, pos, q, k, qo, ko)
    one = torch.empty_like(k)
    psa.psa_rotary(p, spec, pos, None, k, None, one)
    both = (q.clone(), k.clone())
    psa.psa_rotary(p, spec, pos, *both, *both)
    assert torch.equal(one, ko) and torch.equal(both[0], qo) and torch.equal(both[1], ko)
    perm = torch.randperm(N, dtype=torch.int32).cuda()
    perm[5], perm[70] = -1, N
    for inverse in (False, True):
        a, b = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        psa.psa_rotary(p, spec, pos, q, k, a, b, perm=perm, inverse=inverse)
        hit = torch.zeros(N, dtype=torch.bool, device="cuda")
        ok = [i for i in range(N) if i not in (5, 70)]
        hit[perm[ok].long() if inverse else torch.tensor(ok).cuda()] = True
        assert torch.all(a[:, :, ~hit] == 7.0) and torch.all(b[:, :, ~hit] == 7.0)
        assert not torch.any(torch.all(a[:, :, hit] == 7.0, -1))
        if not inverse:
            assert torch.equal(a[:, :, ok], qo[:, :, perm[ok].long()])


def test_inverse_undoes_and_is_the_gradient():
    """R^T R = 1, and <dy, R x> = <R^T dy, x> for every row, in float32; the gradient of a sum against differences."""
    import torch
    N, d = 50, 64
    p = psa.make_params(1, 2, 2, N, d, 64, 64, 1, dtype=psa.PSA_F32)
    spec = psa.make_rotary(d, (12, 10, 10), pairing=1)
    pos = torch.randint(-1000, 1000, (3, N), dtype=torch.int32, generator=torch.Generator().manual_seed(3)).cuda()
    x, dy = rows((1, 2, N, d), "f32", "heads", 1), rows((1, 2, N, d), "f32", "heads", 2)
    turn = lambda t, inverse=False: (lambda o: (psa.psa_rotary(p, spec, pos, t, None, o, None, inverse=inverse), o)[1])(torch.empty_like(t))   # noqa: E731
    back = turn(turn(x), True)
    assert torch.all((back - x).abs() <= 12 * 2.0 ** -24 * 2 * x.abs().amax())
    dx = f64(turn(dy, True))
    assert np.allclose((f64(turn(x)) * f64(dy)).sum(-1), (f64(x) * dx).sum(-1), rtol=0, atol=64 * 6 * 2.0 ** -24 * 30)
    step, h = 0.5, 1
    for c in (0, 5, 31, 40, 63):
        up, down = x.clone(), x.clone()
        up[..., c] += step
        down[..., c] -= step
        slope = ((f64(turn(up)) - f64(turn(down))) * f64(dy)).sum(-1) / (f64(up) - f64(down))[..., c]
        assert np.abs(slope - dx[..., c]).max() <= 4 * 6 * 2.0 ** -24 * 64 * 5 * h


def test_before_the_path_and_behind_its_gradients():
    """Turned and reordered in one pass = turned, then psa_permute_tokens, bit for bit; the attention runs on it; the gradients come back
    the same way; a graph of the whole replays on new inputs."""
    import torch
    grid = (7, 12, 20)
    w = si.small_variant(si.CONFIGS["dit1p3b"], 7 * 12 * 20, Hq=2, Hkv=2).with_(grid=grid)
    T, Hg, W = grid
    gp = gpu_params(oracle_params(w))
    Q, K, V = (to_dev(x, w.dtype) for x in si.generate_qkv(w))
    perm = torch.from_numpy(psa.psa_hilbert_order(T, Hg, W)).cuda()
    n = torch.arange(w.N, device="cuda")
    pos = torch.stack([n // (Hg * W), n // W % Hg, n % W]).to(torch.int32)
    tokens = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (Q, K)]
    spec = psa.make_rotary(w.d, (22, 21, 21), q=tokens[0], k=tokens[1])
    plain = psa.make_rotary(w.d, (22, 21, 21))
    q1, k1, q2, k2, v1 = (torch.empty_like(Q) for _ in range(5))
    psa.psa_rotary(gp, plain, pos, Q, K, q1, k1)
    for a, b in ((q1, q2), (k1, k2)):
        psa.psa_permute_tokens(gp, a, perm, b)
    psa.psa_rotary(gp, spec, pos, *tokens, q1, k1, perm=perm)
    assert torch.equal(q1, q2) and torch.equal(k1, k2)

    buf = Buffers(gp)
    grads = [torch.empty_like(Q) for _ in range(3)]
    back = [torch.empty((1, w.N, 2, w.d), dtype=Q.dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    dO = torch.randn(Q.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(Q.dtype)
    bwd = torch.empty(psa.psa_query_bwd_sizes(gp), dtype=torch.uint8, device="cuda")

    def step():
        psa.psa_rotary(gp, spec, pos, *tokens, q1, k1, perm=perm)
        psa.psa_permute_tokens(gp, V, perm, v1)
        psa.psa_build_pyramid(gp, k1, v1, buf.Kpyr, buf.Vpyr)
        psa.psa_allocate_levels(gp, q1, k1, buf.Kpyr, buf.M, buf.scratch)
        psa.psa_attention_fwd(gp, q1, k1, v1, buf.Kpyr, buf.Vpyr, buf.M, buf.O, buf.scratch, lse=buf.lse)
        psa.psa_attention_bwd(gp, q1, k1, v1, buf.Kpyr, buf.Vpyr, buf.M, buf.O, buf.lse, dO, *grads, bwd)
        psa.psa_rotary(gp, spec, pos, grads[0], grads[1], *back, perm=perm, inverse=True)

    step()
    eager = [x.clone() for x in (buf.O, *back)]
    for g, b in zip(grads, back):
        y = torch.empty_like(g)
        y[:, :, perm.long()] = g
        want = torch.empty_like(g)
        psa.psa_rotary(gp, plain, pos, y, None, want, None, inverse=True)
        assert torch.equal(want, b)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for turn in range(3):
        if turn == 1:
            for x in tokens:
                x.mul_(0.5)
        else:
            for x, y in zip(tokens, (Q, K)):
                x.copy_(y)
        for x in (buf.O, *back):
            x.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        same = all(torch.equal(x, y) for x, y in zip((buf.O, *back), eager))
        assert same == (turn != 1)


def test_binding_refuses():
    import torch
    p = psa.make_params(1, 2, 2, 40, 64, 64, 64, 1)
    spec = psa.make_rotary(64, (12, 10, 10))
    pos = torch.zeros((3, 40), dtype=torch.int32, device="cuda")
    q = rows((1, 2, 40, 64), "bf16", "heads", 1)
    o = torch.empty_like(q)
    good = dict(pos=pos, Qin=q, Kin=q, Qout=o, Kout=torch.empty_like(q))
    for bad in (dict(pos=pos.long()), dict(pos=pos[:2]), dict(pos=pos.cpu()), dict(pos=None), dict(pos=pos.expand(2, 3, 40)), dict(Qin=q.float()), dict(Qin=q[:, :, :39]), dict(Qin=q.cpu()),
                dict(Qin=rows((1, 2, 40, 64), "bf16", "tokens", 1)), dict(Qout=rows((1, 2, 40, 64), "bf16", "tokens", 1)), dict(perm=torch.zeros(39, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            psa.psa_rotary(p, spec, **{**good, **bad})
    with pytest.raises(ValueError):
        psa.make_rotary(64, (12, 10, 10), q=q[..., ::2])
    with pytest.raises(psa.PsaError):
        psa.psa_rotary(p, spec, pos, q, None, o, o)
    psa.psa_rotary(p, spec, **good)
    torch.cuda.synchronize()
