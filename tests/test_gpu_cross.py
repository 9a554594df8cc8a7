"""Cross attention and its gradients against the oracle in 64 bits, element by element, within bounds that follow from the roundings (cross_oracle.py):
types, head sharing, lengths, masks, layouts, what masked places hold, workspaces, streams, graphs."""
import math

import numpy as np
import pytest

from tests import cross_oracle

pytestmark = pytest.mark.gpu

psa = pytest.importorskip("paper_2512_04025_amd")


def params(dtype, B, Hq, Hkv, N, d, **kw):
    return psa.make_params(B, Hq, Hkv, N, d, 128, 64, 1, dtype=psa.PSA_BF16 if dtype == "bf16" else psa.PSA_F32, **kw)


def rows(shape, dtype, layout, seed, offset=0, gain=1.0):
    """[B, H, L, d]: contiguous, token by token, or the middle one of three projections side by side; `offset` elements behind an aligned address."""
    import torch
    B, H, L, d = shape
    wide = {"heads": (B, H, L, d), "tokens": (B, L, H, d), "fused": (B, L, 3 * H, d)}[layout]
    x = torch.randn(int(np.prod(wide)), generator=torch.Generator().manual_seed(seed)) * gain
    flat = torch.zeros(int(np.prod(wide)) + offset, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    flat = flat[offset:].copy_(x).view(wide)
    return flat if layout == "heads" else flat[:, :, :H].transpose(1, 2) if layout == "tokens" else flat[:, :, H:2 * H].transpose(1, 2)


def f64(x):
    return x.double().cpu().numpy()


def scratch(n):
    import torch
    return torch.full((max(n, 256),), 0xff, dtype=torch.uint8, device="cuda")        # (NaN in fp32: nothing is read that was not written)


class Problem:
    def __init__(self, dtype, d, B, Hq, Hkv, N, M, layout="heads", lengths=None, mask=None, offset=0, gain=1.5, seed=0, scale=0.0):
        import torch
        self.dtype, self.p = dtype, params(dtype, B, Hq, Hkv, N, d, scale=scale)
        self.scale = scale or 1 / math.sqrt(d)
        q, k = (B, Hq, N, d), (B, Hkv, M, d)
        self.Q, self.K, self.V = (rows(s, dtype, layout, seed + i, offset, g) for s, i, g in ((q, 1, gain), (k, 2, 1.0), (k, 3, 1.0)))
        self.dO, self.O = rows(q, dtype, layout, seed + 4, offset), rows(q, dtype, layout, seed + 5, offset)
        self.grads = [rows(s, dtype, layout, seed + 6, offset) for s in (q, k, k)]
        self.lse = torch.full((B, Hq, N), 5.0, device="cuda")
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.mask = None if mask is None else torch.as_tensor(mask).to(torch.uint8).cuda()
        self.vis = cross_oracle.visible(B, M, lengths, None if mask is None else np.asarray(mask))
        self.x = psa.make_cross(M, q=self.Q, k=self.K, v=self.V, o=self.O, do=self.dO, dq=self.grads[0], dk=self.grads[1], dv=self.grads[2])
        fwd, bwd = psa.psa_query_cross_sizes(self.p, self.x)
        self.ws = scratch(fwd), scratch(bwd)

    def forward(self, **kw):
        psa.psa_cross_attention_fwd(self.p, self.x, self.Q, self.K, self.V, self.O, self.ws[0], lse=self.lse, kv_len=self.lengths, key_mask=self.mask, **kw)

    def backward(self, **kw):
        psa.psa_cross_attention_bwd(self.p, self.x, self.Q, self.K, self.V, self.O, self.lse, self.dO, *self.grads, self.ws[1], kv_len=self.lengths, key_mask=self.mask, **kw)

    def check(self, backward=True):
        import torch
        self.forward()
        torch.cuda.synchronize()
        Q, K, V = f64(self.Q), f64(self.K), f64(self.V)
        O, lse, bO, bl = cross_oracle.forward(Q, K, V, self.vis, self.scale, self.dtype)
        got = f64(self.lse)
        empty = ~np.isfinite(lse)
        assert np.array_equal(np.isneginf(got), empty)
        assert np.all(np.abs(got[~empty] - lse[~empty]) <= bl[~empty])
        assert np.all(np.abs(f64(self.O) - O) <= bO)
        if not backward:
            return
        self.backward()
        torch.cuda.synchronize()
        want, bound = cross_oracle.backward(Q, K, V, f64(self.O), got, f64(self.dO), self.vis, self.scale, self.dtype)
        for name, g, w, b in zip(("dQ", "dK", "dV"), self.grads, want, bound):
            assert np.all(np.abs(f64(g) - w) <= b), name


BOTH = pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])


@BOTH
@pytest.mark.parametrize("N,M", [(1, 1), (1, 77), (3, 64), (31, 33), (32, 32), (33, 31), (64, 65), (65, 63), (127, 128), (129, 200), (200, 129), (300, 2), (5, 1000)])
def test_lengths(dtype, d, N, M):
    Problem(dtype, d, 1, 2, 2, N, M).check()


@BOTH
@pytest.mark.parametrize("B,Hq,Hkv,N,M", [(2, 7, 1, 1, 70), (3, 8, 2, 5, 130), (2, 6, 3, 50, 96), (1, 28, 4, 33, 65), (1, 4, 2, 130, 513)])
def test_shared_heads_and_layouts(dtype, d, B, Hq, Hkv, N, M):
    Problem(dtype, d, B, Hq, Hkv, N, M, layout="tokens").check()
    Problem(dtype, d, B, Hq, Hkv, N, M, layout="fused", lengths=[M - 1] + [M // 2] * (B - 1)).check()


@BOTH
def test_lengths_and_masks_of_a_batch(dtype, d):
    rng = np.random.default_rng(3)
    M = 150
    mask = rng.random((6, M)) < 0.6
    mask[1] = False                                     # sees nothing
    mask[2, :64], mask[2, 64:128] = True, False         # a tile that is whole, one that is empty
    mask[3, :] = False
    mask[3, 149] = True                                 # the last state alone
    Problem(dtype, d, 6, 4, 2, 70, M, lengths=[150, 100, 150, 150, 0, 1], mask=mask, layout="tokens").check()
    Problem(dtype, d, 5, 2, 2, 40, M, lengths=[-3, 155, 64, 65, 2 ** 31 - 1]).check()
    Problem(dtype, d, 6, 2, 1, 20, M, mask=mask).check()


@BOTH
@pytest.mark.parametrize("hidden", [float("nan"), float("inf"), -float("inf"), "lowest"])
def test_what_hidden_states_hold_does_not_matter(dtype, d, hidden):
    import torch
    rng = np.random.default_rng(4)
    mask = rng.random((2, 200)) < 0.5
    a = Problem(dtype, d, 2, 4, 2, 50, 200, lengths=[180, 120], mask=mask, layout="tokens")
    a.check()
    want = [x.clone() for x in (a.O, a.lse, *a.grads)]
    bad = torch.finfo(a.K.dtype).min if hidden == "lowest" else hidden
    gone = ~torch.from_numpy(a.vis).cuda()
    for x in (a.K, a.V):
        x.copy_(torch.where(gone[:, None, :, None], torch.tensor(bad, dtype=x.dtype, device="cuda"), x))
    a.forward()
    a.backward()
    for x, y in zip((a.O, a.lse, *a.grads), want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,d,B,Hq,Hkv,N,M", [("bf16", 128, 1, 1, 1, 1, 9000), ("bf16", 64, 2, 7, 1, 9, 5003), ("bf16", 128, 1, 2, 2, 100, 3001), ("f32", 64, 1, 2, 1, 30, 3001), ("f32", 128, 2, 2, 2, 1, 2001)])
def test_few_rows_and_many_states_are_shared(dtype, d, B, Hq, Hkv, N, M):
    a = Problem(dtype, d, B, Hq, Hkv, N, M)
    assert psa.psa_query_cross_sizes(a.p, M)[0] > 0
    a.check()
    rng = np.random.default_rng(8)
    mask = rng.random((B, M)) < 0.3
    mask[:, : M // 2] = False                           # whole parts that see nothing
    Problem(dtype, d, B, Hq, Hkv, N, M, layout="tokens", mask=mask, lengths=[M - 7] * B).check()
    Problem(dtype, d, B, Hq, Hkv, N, M, lengths=[0] * (B - 1) + [3]).check()


@pytest.mark.parametrize("dtype,d,B,Hq,Hkv,N,M", [("bf16", 128, 1, 2, 2, 5000, 77), ("bf16", 64, 1, 6, 2, 1501, 130), ("f32", 64, 1, 2, 2, 2001, 40), ("f32", 128, 2, 2, 1, 700, 33)])
def test_many_rows_and_few_states(dtype, d, B, Hq, Hkv, N, M):
    Problem(dtype, d, B, Hq, Hkv, N, M, layout="tokens", lengths=[M - 5] * B).check()


@BOTH
@pytest.mark.parametrize("offset", [1, 3])
def test_element_alignment(dtype, d, offset):
    Problem(dtype, d, 1, 3, 3, 45, 70, layout="fused", offset=offset).check()


@BOTH
def test_offsets_beyond_32_bits(dtype, d):
    """Rows 16 MB apart, 270 of them: every tensor ends 4.5 GB behind its first element."""
    import torch
    a = Problem(dtype, d, 1, 2, 2, 270, 261, lengths=[258])
    esize = a.Q.element_size()
    step = 2 ** 24 // esize
    flat = torch.empty(270 * step, dtype=a.Q.dtype, device="cuda")
    far = [flat.as_strided(x.shape, (270 * step, d, step, 1), i * 2 * d).copy_(x) for i, x in enumerate((a.Q, a.K, a.V, a.O, a.dO, *a.grads))]
    a.Q, a.K, a.V, a.O, a.dO, a.grads = *far[:5], far[5:]
    a.x = psa.make_cross(261, q=a.Q, k=a.K, v=a.V, o=a.O, do=a.dO, dq=a.grads[0], dk=a.grads[1], dv=a.grads[2])
    a.check()


def test_as_many_heads_as_a_call_takes():
    """65535 key heads of one or two rows and few states, float32, against 64 bits on the GPU; one more is refused."""
    import torch
    B, H, N, M, d = 4369, 15, 2, 5, 64
    p = params("f32", B, H, H, N, d)
    gen = torch.Generator("cuda").manual_seed(5)
    Q, K, V, dO = (torch.randn((B, H, n, d), generator=gen, device="cuda") for n in (N, M, M, N))
    O, lse, grads = torch.empty_like(Q), torch.empty((B, H, N), device="cuda"), [torch.empty_like(x) for x in (Q, K, V)]
    x = psa.make_cross(M)
    fwd, bwd = psa.psa_query_cross_sizes(p, x)
    psa.psa_cross_attention_fwd(p, x, Q, K, V, O, scratch(fwd), lse=lse)
    psa.psa_cross_attention_bwd(p, x, Q, K, V, O, lse, dO, *grads, scratch(bwd))
    q, k, v, g, o = (t.double() for t in (Q, K, V, dO, O))
    s = (q[:, :, :, None] * k[:, :, None]).sum(-1) / 8
    w = torch.softmax(s, -1)
    # a score is off by its 64 products and sums, the rest by fewer than 40 roundings of its terms
    u = 2.0 ** -24
    delta = u * ((d + 4) * (q.abs()[:, :, :, None] * k.abs()[:, :, None]).sum(-1).max() / 8 + 8 * (1 + s.abs().max()))
    assert torch.all((lse.double() - torch.logsumexp(s, -1)).abs() <= delta + 40 * u)
    want, size = ((w[..., None] * t[:, :, None]).sum(3) for t in (v, v.abs()))
    assert torch.all((o - want).abs() <= size * (2 * delta + 40 * u))
    p_ = torch.exp(s - lse.double()[..., None])
    dv, size = ((p_[..., None] * t[:, :, :, None]).sum(2) for t in (g, g.abs()))
    assert torch.all((grads[2].double() - dv).abs() <= size * (2 * delta + 40 * u))
    with pytest.raises(psa.PsaError):
        psa.psa_query_cross_sizes(params("f32", B + 1, H, H, N, d), x)


def test_states_beyond_the_cache():
    """A row or three against 300 MB of states, lengths that end in the last part: against 64 bits on the GPU, a head at a time."""
    import torch
    H, N, M, d, length = 2, 3, 300000, 128, 299990
    p = params("bf16", 1, H, H, N, d)
    Q, K, V = (torch.randn((1, H, n, d), generator=torch.Generator("cuda").manual_seed(n + i), device="cuda").to(torch.bfloat16) for i, n in ((1, N), (2, M), (3, M)))
    O, lse = torch.empty_like(Q), torch.empty((1, H, N), device="cuda")
    x = psa.make_cross(M)
    psa.psa_cross_attention_fwd(p, x, Q, K, V, O, scratch(psa.psa_query_cross_sizes(p, x)[0]), lse=lse, kv_len=torch.tensor([length], dtype=torch.int32, device="cuda"))
    for h in range(H):
        q, k, v = Q[0, h].double(), K[0, h, :length].double(), V[0, h, :length].double()
        s = q @ k.t().contiguous() / math.sqrt(d)
        w = torch.softmax(s, 1)
        # 128 products and a scale in 32 bits are the error of a score, the states' sums that of the rest; weights and outputs are rounded to bfloat16
        delta = 2.0 ** -24 * ((d + 4) * (q.abs() @ k.abs().t().contiguous()).max() / math.sqrt(d) + 8 * (1 + s.abs().max()))
        assert torch.all((lse[0, h].double() - torch.logsumexp(s, 1)).abs() <= delta + (M + 60) * 2.0 ** -24)
        assert torch.all((O[0, h].double() - w @ v).abs() <= 1.01 * ((w @ v.abs()) * (2.0 ** -8 + 2 * delta + (M + 8) * 2.0 ** -24) + 2.0 ** -8 * (w @ v).abs()))


@BOTH
def test_scores_of_a_wide_range(dtype, d):
    """A softmax that one state takes, and a scale of the caller's."""
    Problem(dtype, d, 1, 2, 2, 70, 300, gain=20.0).check()
    Problem(dtype, d, 1, 2, 2, 70, 300, scale=0.7).check()


@BOTH
def test_growing_scores_move_the_maximum(dtype, d):
    import torch
    a = Problem(dtype, d, 1, 1, 1, 64, 640)
    ramp = torch.linspace(0.0, 6.0, 640, device="cuda")[None, None, :, None]
    a.Q.copy_(a.Q.abs())
    a.K.copy_(a.K.abs() * ramp)
    a.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_states(dtype):
    import torch
    for K in (None, torch.empty((2, 2, 0, 64), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")):
        p = params(dtype, 2, 4, 2, 37, 64)
        q = rows((2, 4, 37, 64), dtype, "heads", 1)
        O, dQ, lse = torch.ones_like(q), torch.ones_like(q), torch.ones((2, 4, 37), device="cuda")
        x = psa.make_cross(0)
        psa.psa_cross_attention_fwd(p, x, q, K, K, O, None, lse=lse)
        psa.psa_cross_attention_bwd(p, x, q, K, K, O, lse, q, dQ, K, K, scratch(psa.psa_query_cross_sizes(p, x)[1]))
        assert torch.all(O == 0) and torch.all(torch.isneginf(lse)) and torch.all(dQ == 0)


def test_states_that_a_batch_shares():
    """Stride 0 over the batch on the way in; every entry's gradient on the way out."""
    import torch
    a = Problem("bf16", 64, 3, 4, 2, 50, 90)
    one = a.K[:1].clone(), a.V[:1].clone()
    a.K.copy_(one[0].expand_as(a.K))
    a.V.copy_(one[1].expand_as(a.V))
    a.check()
    want = [x.clone() for x in (a.O, *a.grads)]
    K, V = (t.expand(3, -1, -1, -1) for t in one)
    x = psa.make_cross(90, k=K, v=V)
    psa.psa_cross_attention_fwd(a.p, x, a.Q, K, V, a.O, a.ws[0], lse=a.lse)
    psa.psa_cross_attention_bwd(a.p, x, a.Q, K, V, a.O, a.lse, a.dO, *a.grads, a.ws[1])
    assert all(torch.equal(u, v) for u, v in zip((a.O, *a.grads), want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_else_is_written(dtype):
    """Outputs side by side with other projections, and rows of memory before and behind them, keep what they held."""
    import torch
    a = Problem(dtype, 64, 2, 4, 2, 75, 101, layout="fused", lengths=[101, 30])
    outs = [a.O, *a.grads]
    bases = [x._base if x._base is not None else x for x in outs]
    for x, base in zip(outs, bases):
        base.fill_(7.0)
    a.check()
    for x, base in zip(outs, bases):
        x.fill_(7.0)
        assert torch.all(base == 7.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_and_nan_inputs_stay_in_their_rows(dtype):
    """A query row that is not finite spoils its own output alone; a state's value that is not finite, its channel alone."""
    import torch
    a = Problem(dtype, 64, 1, 2, 2, 70, 100)
    a.forward()
    clean = a.O.clone()
    a.Q[0, 1, 33, 5] = float("nan")
    a.V[0, 0, 40, 9] = float("inf")
    a.forward()
    bad = torch.isnan(a.O)
    assert torch.all(bad[0, 1, 33]) and bad.sum() == 64
    assert torch.all(torch.isinf(a.O[0, 0, :, 9]))
    same = ~bad
    same[0, 0, :, 9] = False
    assert torch.equal(a.O[same], clean[same])


def test_a_row_that_is_not_finite_spoils_its_own_parts():
    """The same where workgroups share the states."""
    import torch
    for dtype in ("bf16", "f32"):
        a = Problem(dtype, 64, 1, 1, 1, 40, 5000)
        assert psa.psa_query_cross_sizes(a.p, 5000)[0] > 0
        a.forward()
        clean = a.O.clone()
        a.Q[0, 0, 7, 5] = float("nan")
        a.forward()
        assert torch.all(torch.isnan(a.O[0, 0, 7])) and torch.isnan(a.lse[0, 0, 7])
        ok = [i for i in range(40) if i != 7]
        assert torch.equal(a.O[:, :, ok], clean[:, :, ok])


@pytest.mark.parametrize("dtype,N,M", [("bf16", 300, 200), ("bf16", 4, 4000), ("f32", 130, 90)])
def test_bits_repeat_on_other_streams_and_in_graphs(dtype, N, M):
    import torch
    a, b = (Problem(dtype, 128, 1, 4, 2, N, M, lengths=[M - 3], seed=s) for s in (0, 50))
    for x in (a, b):
        x.check()
    want = [[t.clone() for t in (x.O, x.lse, *x.grads)] for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):                                  # two at once, each with its own workspace
        for x, s in zip((a, b), streams):
            x.forward(stream=s)
            x.backward(stream=s)
    torch.cuda.synchronize()
    for x, w in zip((a, b), want):
        assert all(torch.equal(u, v) for u, v in zip((x.O, x.lse, *x.grads), w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        a.forward()
        a.backward()
    keep = a.Q.clone()
    for turn in range(3):
        a.Q.copy_(keep * (0.5 if turn == 1 else 1.0))
        for t in (a.O, a.lse, *a.grads):
            t.fill_(3.0)
        graph.replay()
        b.forward()
        torch.cuda.synchronize()
        got = [t.clone() for t in (a.O, a.lse, *a.grads)]
        a.forward()
        a.backward()
        assert all(torch.equal(u, v) for u, v in zip(got, (a.O, a.lse, *a.grads)))
        assert all(torch.equal(u, v) for u, v in zip(got, want[0])) == (turn != 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_graphs_share_a_workspace(dtype):
    """Problems of other sizes whose calls leave partial results in the same memory, replayed by turns on one stream, with an eager call between."""
    import torch
    a, b = Problem(dtype, 64, 1, 2, 2, 20, 3000, seed=3), Problem(dtype, 64, 2, 2, 1, 700, 150, lengths=[150, 9], seed=60)
    shared = [scratch(max(x.ws[i].numel() for x in (a, b))) for i in (0, 1)]
    graphs, want = [], []
    for x in (a, b):
        x.check()
        want.append([t.clone() for t in (x.O, x.lse, *x.grads)])
        x.ws = shared
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            x.forward()
            x.backward()
    for turn in (0, 1, 1, 0, 1, 0):
        x = (a, b)[turn]
        for t in (x.O, x.lse, *x.grads):
            t.fill_(3.0)
        graphs[turn].replay()
        (b, a)[turn].forward()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip((x.O, x.lse, *x.grads), want[turn]))


def test_gradients_against_differences():
    """float32: (f(x + h) - f(x - h)) / 2h of <O, dO> summed in 64 bits. The outputs are off by at most bO, so the slope by sum bO |dO| / h, and by h^2 / 6 times a third
    derivative, for which 50 stands (inputs of size one, 12 states)."""
    import torch
    a = Problem("f32", 64, 1, 2, 1, 5, 12, gain=1.0)
    a.forward()
    a.backward()
    grads = [f64(g) for g in a.grads]
    rng = np.random.default_rng(1)
    h = 2.0 ** -5
    for x, g in zip((a.Q, a.K, a.V), grads):
        for at in [tuple(int(rng.integers(0, n)) for n in x.shape) for _ in range(8)]:
            keep, f = x[at].item(), []
            for sign in (1, -1):
                x[at] = keep + sign * h
                a.forward()
                f.append((f64(a.O) * f64(a.dO)).sum())
                _, _, bO, _ = cross_oracle.forward(f64(a.Q), f64(a.K), f64(a.V), a.vis, a.scale, "f32")
            x[at] = keep
            assert abs((f[0] - f[1]) / (2 * h) - g[at]) <= (bO * np.abs(f64(a.dO))).sum() / h + 50 * h * h / 6


def test_a_layer_of_the_whole():
    """Rotary positions and Hilbert order, pyramid attention, its output as the queries of the cross attention, and the gradients of both behind one
    another; captured into a graph, replayed on other inputs and back."""
    import torch
    from tests.psa_testlib import Buffers
    T, Hg, W, H, d, M = 5, 12, 16, 4, 128, 77
    N = T * Hg * W
    gp = psa.make_params(1, H, H, N, d, 128, 64, 3, budget=0.5)
    tokens = [rows((1, H, N, d), "bf16", "tokens", i) for i in range(3)]
    text = [rows((1, H, M, d), "bf16", "tokens", 10 + i) for i in range(2)]
    dO = rows((1, H, N, d), "bf16", "heads", 20)
    n = torch.arange(N, device="cuda")
    pos = torch.stack([n // (Hg * W), n // W % Hg, n % W]).to(torch.int32)
    perm = torch.from_numpy(psa.psa_hilbert_order(T, Hg, W)).cuda()
    lens = torch.tensor([60], dtype=torch.int32, device="cuda")
    spec = psa.make_rotary(d, (22, 21, 21), q=tokens[0], k=tokens[1])
    x = psa.make_cross(M, k=text[0], v=text[1])
    buf = Buffers(gp)
    new = lambda like: torch.empty(like.shape, dtype=like.dtype, device="cuda")      # noqa: E731
    q, k, v, co, dq_c, dq, dk, dv = (new(dO) for _ in range(8))
    dkt, dvt, back = new(text[0]), new(text[0]), [torch.empty((1, N, H, d), dtype=dO.dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    lse = torch.empty((1, H, N), device="cuda")
    fwd, bwd = psa.psa_query_cross_sizes(gp, x)
    wsf, wsb, wsp = scratch(fwd), scratch(bwd), scratch(psa.psa_query_bwd_sizes(gp))

    def layer():
        psa.psa_rotary(gp, spec, pos, tokens[0], tokens[1], q, k, perm=perm)
        psa.psa_permute_tokens(gp, tokens[2].contiguous(), perm, v)
        psa.psa_build_pyramid(gp, k, v, buf.Kpyr, buf.Vpyr)
        psa.psa_allocate_levels(gp, q, k, buf.Kpyr, buf.M, buf.scratch)
        psa.psa_attention_fwd(gp, q, k, v, buf.Kpyr, buf.Vpyr, buf.M, buf.O, buf.scratch, lse=buf.lse)
        psa.psa_cross_attention_fwd(gp, x, buf.O, *text, co, wsf, lse=lse, kv_len=lens)
        psa.psa_cross_attention_bwd(gp, x, buf.O, *text, co, lse, dO, dq_c, dkt, dvt, wsb, kv_len=lens)
        psa.psa_attention_bwd(gp, q, k, v, buf.Kpyr, buf.Vpyr, buf.M, buf.O, buf.lse, dq_c, dq, dk, dv, wsp)
        psa.psa_rotary(gp, spec, pos, dq, dk, *back, perm=perm, inverse=True)
        return [co, dkt, dvt, *back]

    want = [t.clone() for t in layer()]
    assert all(torch.all(torch.isfinite(t)) for t in want)
    vis = cross_oracle.visible(1, M, [60], None)
    args = [f64(t) for t in (buf.O, *text)]
    O, l, bO, bl = cross_oracle.forward(*args, vis, 1 / math.sqrt(d), "bf16")
    assert np.all(np.abs(f64(co) - O) <= bO) and np.all(np.abs(f64(lse) - l) <= bl)
    grads, bounds = cross_oracle.backward(*args, f64(co), f64(lse), f64(dO), vis, 1 / math.sqrt(d), "bf16")
    for g, w, b in zip((dq_c, dkt, dvt), grads, bounds):
        assert np.all(np.abs(f64(g) - w) <= b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        out = layer()
    keep = [t.clone() for t in tokens]
    for turn in range(3):
        for t, y in zip(tokens, keep):
            t.copy_(y * (0.75 if turn == 1 else 1.0))
        for t in out:
            t.fill_(1.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(u, v) for u, v in zip(got, layer()))
        assert all(torch.equal(u, v) for u, v in zip(got, want)) == (turn != 1)


def test_binding_refuses():
    import torch
    a = Problem("bf16", 64, 2, 4, 2, 40, 50, lengths=[50, 20], mask=np.ones((2, 50)))
    good = dict(p=a.p, x=a.x, Q=a.Q, K=a.K, V=a.V, O=a.O, scratch=a.ws[0], lse=a.lse, kv_len=a.lengths, key_mask=a.mask)
    for bad in (dict(Q=a.Q[:, :, :39]), dict(Q=a.Q.float()), dict(Q=a.Q.cpu()), dict(K=a.K[:, :, :49]), dict(K=a.Q), dict(V=rows((2, 2, 50, 64), "bf16", "tokens", 1)), dict(lse=a.lse.double()),
                dict(kv_len=a.lengths.long()), dict(kv_len=a.lengths[:1]), dict(key_mask=a.mask[:, :49]), dict(key_mask=a.mask.float()), dict(key_mask=a.mask.cpu()), dict(O=a.O[..., :32])):
        with pytest.raises(ValueError):
            psa.psa_cross_attention_fwd(**{**good, **bad})
    with pytest.raises(ValueError):
        psa.psa_cross_attention_bwd(a.p, a.x, a.Q, a.K, a.V, a.O, a.lse, a.dO, *a.grads, a.ws[1][:64])
    with pytest.raises(psa.PsaError):
        psa.psa_cross_attention_fwd(**{**good, "Q": None})
    with pytest.raises(ValueError):
        psa.make_cross(50, q=a.Q[..., ::2])
    few = Problem("bf16", 64, 1, 1, 1, 1, 9000)
    with pytest.raises(ValueError):
        psa.psa_cross_attention_fwd(few.p, few.x, few.Q, few.K, few.V, few.O, None)
    psa.psa_cross_attention_fwd(**{**good, "key_mask": a.mask.bool()})
    torch.cuda.synchronize()
