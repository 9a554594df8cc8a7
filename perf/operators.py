"""What is timed of the operators around the pyramid attention: rotary positions with several axes, which turn Q and
K before it (and the gradients back behind it), and cross attention to an encoder's states of another length.

A case is one pass
    rotary          Q and K from the projections' layout, turned by their positions on the axes of the token grid,
                    in the order of a permutation where one is given
    rotary_grad     the same backwards: what the gradients of the turned Q and K are for the projections
    cross           attention of N query tokens to M encoder states, with the softmax statistics
    cross_grad      gradients of Q, K and V
With `own` false the passes are elementary torch operations in 32 bits (angles in 64), with `own` true they are the
package's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

BASE = 10000.0


# ---------------------------------------------------------------------------------------------- cases
def _rotary(name, what, B, Hq, Hkv, N, d, **kw):
    c = dict(what=what, B=B, Hq=Hq, Hkv=Hkv, N=N, d=d, dtype="bf16", pairing="adjacent", shared=False, per_batch=False, T=0, Hg=0, W=0,
             layout="tokens", reorder=False)
    if name:
        c["name"] = name
    c.update(kw)
    return c


def _cross(name, what, B, Hq, Hkv, N, M, d, **kw):
    c = dict(what=what, B=B, Hq=Hq, Hkv=Hkv, N=N, M=M, d=d, dtype="bf16", layout="tokens", lengths=False, mask=False)
    if name:
        c["name"] = name
    c.update(kw)
    return c


def listed():
    return [
        # the next token of eight conversations with a video language model: the smallest call, nothing but latency
        _rotary("rotary_token", "rotary", 8, 28, 4, 1, 128, pairing="halves", shared=True, per_batch=True, layout="heads"),
        # the tiny float32 configuration that results are checked in
        _rotary("rotary_f32_tiny", "rotary", 1, 2, 2, 1024, 64, dtype="f32", layout="heads", T=4, Hg=16, W=16),
        # a layer of the 1.3B video transformer: Q and K as the projections leave them, turned and put in Hilbert order
        _rotary("rotary_dit1p3b", "rotary", 1, 12, 12, 32760, 128, T=21, Hg=30, W=52, reorder=True),
        # training the 14B video transformer: the largest pass over Q and K, back to the projections' layout
        _rotary("rotary_dit14b_grad", "rotary_grad", 1, 40, 40, 75600, 128, T=21, Hg=45, W=80, reorder=True),
        # one token of each of eight sequences against encoded frames, seven query heads to a key head
        _cross("cross_token", "cross", 8, 28, 4, 1, 1500, 128, layout="heads", lengths=True),
        # float32: a short clip against a prompt of 77 tokens, and gradients with an odd, masked prompt
        _cross("cross_f32_clip", "cross", 1, 2, 2, 1024, 77, 64, dtype="f32", layout="heads"),
        _cross("cross_f32_grad", "cross_grad", 1, 12, 12, 1000, 301, 128, dtype="f32", mask=True),
        # the text of a 1.3B video transformer's layer (512 states), and its training step on a padded batch
        _cross("cross_dit1p3b", "cross", 1, 12, 12, 32760, 512, 128),
        _cross("cross_dit1p3b_grad", "cross_grad", 2, 12, 12, 16380, 512, 128, lengths=True),
        # the largest: the 14B video transformer
        _cross("cross_dit14b", "cross", 1, 40, 40, 75600, 512, 128),
        # 64 learned queries that gather a whole video's tokens, and their gradients: few rows, many keys
        _cross("cross_latents", "cross", 2, 16, 16, 64, 32760, 64, mask=True),
        _cross("cross_latents_grad", "cross_grad", 2, 16, 16, 64, 8190, 64, lengths=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more pass of these ranges, with odd lengths."""
    f32 = rng.random() < 0.25
    d = rng.choice([64, 128, 128])
    B, Hq, Hkv = rng.choice([(1, 2, 2), (1, 12, 12), (2, 4, 4), (1, 8, 2), (1, 28, 4), (4, 16, 16), (8, 28, 4), (1, 40, 40)])
    dtype, layout = "f32" if f32 else "bf16", rng.choice(["tokens", "tokens", "heads"])
    if rng.random() < 0.4:
        what = rng.choice(["rotary", "rotary", "rotary_grad"])
        N = _log(rng, 1, 60000)
        c = _rotary(None, what, B, Hq, Hkv, N, d, dtype=dtype, layout=layout, pairing=rng.choice(["adjacent", "halves"]), shared=rng.random() < 0.4,
                    per_batch=rng.random() < 0.3, reorder=rng.random() < 0.4)
        most, size, key = 1.2e9, lambda: work(c)["bytes"], "N"
    else:
        what = rng.choice(["cross", "cross", "cross_grad"])
        c = _cross(None, what, B, Hq, Hkv, _log(rng, 1, 60000), _log(rng, 1, 2000), d, dtype=dtype, layout=layout, lengths=rng.random() < 0.4, mask=rng.random() < 0.3)
        if rng.random() < 0.25:                      # few queries, many states
            c["N"], c["M"] = _log(rng, 1, 128), _log(rng, 1000, 40000)
        most, size, key = (4e10 if f32 else 4e11), lambda: work(c)["flops"], "N"
    while size() > most:
        key = "N" if c["N"] >= c.get("M", 0) else "M"
        c[key] = c[key] * 2 // 3
    return c


# ---------------------------------------------------------------------------------------------- inputs
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _tensor(c, heads, n, gen, gain=1.0):
    """[B, heads, n, d]: stored head by head, or token by token as a projection leaves it."""
    shape = (c["B"], heads, n, c["d"]) if c["layout"] == "heads" else (c["B"], n, heads, c["d"])
    x = torch.randn(shape, generator=gen, device="cuda").mul_(gain).to(_dtype(c))
    return x if c["layout"] == "heads" else x.transpose(1, 2)


def _pairs(c):
    """Channel pairs that turn with t, y and x."""
    half = c["d"] // 2
    if c["shared"]:
        return (half // 4, 3 * half // 8, 3 * half // 8)
    side = half // 3
    return (half - 2 * side, side, side)


def _positions(c, gen):
    """[B or 1, 3, N]: the raster of the token grid, or text and frames with an offset a sequence as a decoder meets them."""
    N = c["N"]
    n = torch.arange(N, device="cuda")
    if c["T"]:
        pos = torch.stack([n // (c["Hg"] * c["W"]), n // c["W"] % c["Hg"], n % c["W"]])[None]
    else:
        side = max(1, int(round(N ** (1 / 3))))
        pos = torch.stack([n // (side * side), n // side % side, n % side])[None]
    if c["per_batch"]:
        pos = pos + torch.randint(0, 30000, (c["B"], 1, 1), generator=gen, device="cuda")
    else:
        pos = pos + torch.randint(0, 100, (1, 1, 1), generator=gen, device="cuda")
    return pos.to(torch.int32).contiguous()


def _frequencies(c):
    """Axis and radians a position of every channel pair, the latter in 64 bits."""
    pairs = _pairs(c)
    axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    if c["shared"]:
        freq = [BASE ** (-i / (c["d"] // 2)) for i in range(c["d"] // 2)]
    else:
        freq = [BASE ** (-i / n) for n in pairs for i in range(n)]
    return axis, freq


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    B, Hq, Hkv, N, d = c["B"], c["Hq"], c["Hkv"], c["N"], c["d"]
    if c["what"].startswith("rotary"):
        s["pos"] = _positions(c, gen)
        axis, freq = _frequencies(c)
        s["axis"], s["freq"] = torch.tensor(axis, device="cuda"), torch.tensor(freq, dtype=torch.float64, device="cuda")
        s["perm"] = torch.randperm(N, generator=gen, device="cuda").to(torch.int32) if c["reorder"] else None
        heads = dict(c, layout="heads")
        back = c["what"] == "rotary_grad"
        s["in"] = [_tensor(heads if back else c, h, N, gen) for h in (Hq, Hkv)]
    else:
        s["Q"], s["K"], s["V"] = _tensor(c, Hq, N, gen, 1.5), _tensor(c, Hkv, c["M"], gen), _tensor(c, Hkv, c["M"], gen)
        s["len"] = s["mask"] = None
        if c["lengths"]:
            s["len"] = torch.randint(c["M"] // 2, c["M"] + 1, (B,), generator=gen, device="cuda").to(torch.int32)
        if c["mask"]:
            s["mask"] = (torch.rand((B, c["M"]), generator=gen, device="cuda") < 0.75).to(torch.uint8)
        if c["what"] == "cross_grad":
            s["dO"] = _tensor(c, Hq, N, gen)
            O, s["lse"] = _cross_plain(s)              # what the forward pass left behind
            s["O"] = torch.empty_like(s["Q"]).copy_(O)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program makes once: parameters, outputs, workspace."""
    import paper_2512_04025_amd as psa
    c = s["case"]
    B, Hq, Hkv, N, d = c["B"], c["Hq"], c["Hkv"], c["N"], c["d"]
    s["p"] = p = psa.make_params(B, Hq, Hkv, N, d, 128, 64, 4, dtype=psa.PSA_BF16 if c["dtype"] == "bf16" else psa.PSA_F32)
    if c["what"].startswith("rotary"):
        back = c["what"] == "rotary_grad"
        rows = (lambda h: torch.empty((B, N, h, d), dtype=_dtype(c), device="cuda").transpose(1, 2)) if back and c["layout"] == "tokens" else (
            lambda h: torch.empty((B, h, N, d), dtype=_dtype(c), device="cuda"))
        s["out"] = [rows(Hq), rows(Hkv)]
        q, k = s["out"] if back else s["in"]
        s["spec"] = psa.make_rotary(d, _pairs(c), base=BASE, shared=c["shared"],
                                    pairing=psa.PSA_ROTARY_ADJACENT if c["pairing"] == "adjacent" else psa.PSA_ROTARY_HALVES, q=q, k=k)
        return
    forward, backward = psa.psa_query_cross_sizes(p, c["M"])
    if c["what"] == "cross":
        s["out"] = [torch.empty_like(s["Q"]), torch.empty((B, Hq, N), dtype=torch.float32, device="cuda")]
        s["spec"] = psa.make_cross(c["M"], q=s["Q"], k=s["K"], v=s["V"], o=s["out"][0])
        s["scratch"] = torch.empty(max(forward, 256), dtype=torch.uint8, device="cuda")
    else:
        s["out"] = [torch.empty_like(s[n]) for n in "QKV"]
        s["spec"] = psa.make_cross(c["M"], q=s["Q"], k=s["K"], v=s["V"], o=s["O"], do=s["dO"], dq=s["out"][0], dk=s["out"][1], dv=s["out"][2])
        s["scratch"] = torch.empty(max(backward, 256), dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s)
    if c["what"] == "rotary":
        return dict(zip(("Q", "K"), _rotary_plain(s)))
    if c["what"] == "rotary_grad":
        return dict(zip(("dQ", "dK"), _rotary_plain(s)))
    if c["what"] == "cross":
        return dict(zip(("O", "lse"), _cross_plain(s)))
    return dict(zip(("dQ", "dK", "dV"), _cross_grad_plain(s)))


def _own(s):
    import paper_2512_04025_amd as psa
    c, out = s["case"], s["out"]
    if c["what"] == "rotary":
        psa.psa_rotary(s["p"], s["spec"], s["pos"], *s["in"], *out, perm=s["perm"])
        return {"Q": out[0], "K": out[1]}
    if c["what"] == "rotary_grad":
        psa.psa_rotary(s["p"], s["spec"], s["pos"], *s["in"], *out, perm=s["perm"], inverse=True)
        return {"dQ": out[0], "dK": out[1]}
    if c["what"] == "cross":
        psa.psa_cross_attention_fwd(s["p"], s["spec"], s["Q"], s["K"], s["V"], out[0], s["scratch"], lse=out[1], kv_len=s["len"], key_mask=s["mask"])
        return {"O": out[0], "lse": out[1]}
    psa.psa_cross_attention_bwd(s["p"], s["spec"], s["Q"], s["K"], s["V"], s["O"], s["lse"], s["dO"], *out, s["scratch"], kv_len=s["len"], key_mask=s["mask"])
    return {"dQ": out[0], "dK": out[1], "dV": out[2]}


def _rotary_plain(s):
    c = s["case"]
    angle = s["pos"].double()[:, s["axis"]].transpose(1, 2) * s["freq"]           # [B or 1, N, d / 2]
    back = c["what"] == "rotary_grad"
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    sin = -sin if back else sin
    return _rounded(c, *(_turn(x, cos, sin, c["pairing"], s["perm"], back) for x in s["in"]))


def _turn(x, cos, sin, pairing, perm, back):
    if perm is not None and back:
        y = torch.empty_like(x)
        y[:, :, perm.long()] = x
        x = y
    elif perm is not None:
        x, cos, sin = x[:, :, perm.long()], cos[:, :, perm.long()], sin[:, :, perm.long()]
    half = x.shape[-1] // 2
    x = x.float()
    x0, x1 = (x[..., 0::2], x[..., 1::2]) if pairing == "adjacent" else (x[..., :half], x[..., half:])
    y0, y1 = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    y = torch.stack([y0, y1], -1).flatten(-2) if pairing == "adjacent" else torch.cat([y0, y1], -1)
    return y


def _rounded(c, *xs):
    return [x.to(_dtype(c)) for x in xs]


def _visible(s):
    """[B, 1, 1, M]: which states a query sees; None where it sees all."""
    c, vis = s["case"], None
    if s["len"] is not None:
        vis = torch.arange(c["M"], device="cuda") < s["len"][:, None]
    if s["mask"] is not None:
        vis = s["mask"].bool() if vis is None else vis & s["mask"].bool()
    return None if vis is None else vis[:, None, None]


def _grouped(s, x):
    """Query heads of one key head as rows of one matrix: [B, Hkv, group N, d], in 32 bits."""
    c = s["case"]
    return x.float().reshape(c["B"], c["Hkv"], -1, x.shape[-1])


def _keys(s, x, vis):
    x = x.float()
    return x if vis is None else torch.where(vis.transpose(2, 3), x, 0.0)


def _scores(s, q, k, vis):
    x = (q @ k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(s["case"]["d"]))
    return x if vis is None else x.masked_fill_(~vis, -math.inf)


def _cross_plain(s):
    c, vis = s["case"], _visible(s)
    x = _scores(s, _grouped(s, s["Q"]), _keys(s, s["K"], vis), vis)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    O = (p @ _keys(s, s["V"], vis)) / torch.where(total == 0, 1.0, total)
    O, lse = O.reshape(c["B"], c["Hq"], c["N"], c["d"]), (top + torch.log(total)).reshape(c["B"], c["Hq"], c["N"])
    return _rounded(c, O)[0], lse


def _cross_grad_plain(s):
    c, vis, scale = s["case"], _visible(s), 1.0 / math.sqrt(s["case"]["d"])
    q, g, o = _grouped(s, s["Q"]), _grouped(s, s["dO"]), _grouped(s, s["O"])
    k, v = _keys(s, s["K"], vis), _keys(s, s["V"], vis)
    lse = s["lse"].reshape(c["B"], c["Hkv"], -1, 1)
    p = _scores(s, q, k, vis).sub_(torch.where(torch.isinf(lse), 0.0, lse)).exp_()
    dv = p.transpose(2, 3).contiguous() @ g
    ds = p.mul_((g @ v.transpose(2, 3).contiguous()).sub_((g * o).sum(-1, keepdim=True))).mul_(scale)
    dq = (ds @ k).reshape(c["B"], c["Hq"], c["N"], c["d"])
    return _rounded(c, dq, ds.transpose(2, 3).contiguous() @ q, dv)


# ---------------------------------------------------------------------------------------------- what it takes
def work(case):
    """Every input read once, every output written once; FLOPs of the products with the states that are seen (a length is
    three quarters of M on average, as is a mask's share), five for the gradients and two for the output."""
    c = case
    e, B, N, d = (2 if c["dtype"] == "bf16" else 4), c["B"], c["N"], c["d"]
    if c["what"].startswith("rotary"):
        n = B * (c["Hq"] + c["Hkv"]) * N * d
        return {"bytes": 2 * n * e + 12 * N * (B if c["per_batch"] else 1) + (4 * N if c["reorder"] else 0), "flops": 3 * n}
    seen = c["M"] * (0.75 if c["lengths"] else 1.0) * (0.75 if c["mask"] else 1.0)
    q, k, products = B * c["Hq"] * N * d, B * c["Hkv"] * c["M"] * (0.75 if c["lengths"] else 1.0) * d, 2.0 * B * c["Hq"] * N * seen * d
    if c["what"] == "cross":
        return {"bytes": int(e * (2 * q + 2 * k) + 4 * q / d), "flops": 2 * products}
    return {"bytes": int(e * (4 * q + 2 * k + 2 * B * c["Hkv"] * c["M"] * d) + 4 * q / d), "flops": 5 * products}


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """The definitions in 64 bits, a head at a time."""
    s = prepare(case, seed)
    if case["what"].startswith("rotary"):
        return _rotary_exact(case, s)
    c = case
    B, Hq, Hkv, N, M, d = c["B"], c["Hq"], c["Hkv"], c["N"], c["M"], c["d"]
    new = lambda h, n: torch.zeros((B, h, n, d), dtype=torch.float64, device="cuda")     # noqa: E731
    O, lse, dQ, dK, dV = new(Hq, N), torch.zeros((B, Hq, N), dtype=torch.float64, device="cuda"), new(Hq, N), new(Hkv, M), new(Hkv, M)
    for b in range(B):
        seen = torch.ones(M, dtype=torch.bool, device="cuda")
        if s["len"] is not None:
            seen[int(s["len"][b]):] = False
        if s["mask"] is not None:
            seen &= s["mask"][b] != 0
        j = torch.nonzero(seen)[:, 0]
        if not len(j):
            lse[b] = -math.inf
            continue
        for h in range(Hq):
            hk = h // (Hq // Hkv)
            q, k, v = s["Q"][b, h].double(), s["K"][b, hk, j].double(), s["V"][b, hk, j].double()
            z = torch.mm(q, k.t().contiguous()) / math.sqrt(d)
            if c["what"] == "cross":
                lse[b, h] = torch.logsumexp(z, 1)
                O[b, h] = torch.mm(torch.softmax(z, 1), v)
                continue
            g = s["dO"][b, h].double()
            w = torch.exp(z - s["lse"][b, h].double()[:, None])
            e = w * (torch.mm(g, v.t().contiguous()) - (g * s["O"][b, h].double()).sum(1)[:, None]) / math.sqrt(d)
            dQ[b, h] = torch.mm(e, k)
            dK[b, hk].index_add_(0, j, torch.mm(e.t().contiguous(), q))
            dV[b, hk].index_add_(0, j, torch.mm(w.t().contiguous(), g))
    return {"O": O, "lse": lse} if c["what"] == "cross" else {"dQ": dQ, "dK": dK, "dV": dV}


def _rotary_exact(c, s):
    """Every pair as a complex number, turned by exp(i angle)."""
    half = c["d"] // 2
    back = c["what"] == "rotary_grad"
    angle = s["pos"].double().index_select(1, s["axis"]) * s["freq"][:, None]      # [B or 1, d / 2, N]
    turn = torch.polar(torch.ones_like(angle), -angle if back else angle).transpose(1, 2)
    out = []
    for x in s["in"]:
        y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for b in range(c["B"]):
            w = turn[b if c["per_batch"] else 0]
            for h in range(x.shape[1]):
                src = x[b, h].double()
                if s["perm"] is not None:
                    to = s["perm"].long()
                    if back:
                        src = src[torch.argsort(to)]
                    else:
                        src = src[to]
                z = torch.complex(src[:, 0::2], src[:, 1::2]) if c["pairing"] == "adjacent" else torch.complex(src[:, :half], src[:, half:])
                z = z * (w if s["perm"] is None or back else w[to])
                if c["pairing"] == "adjacent":
                    y[b, h, :, 0::2], y[b, h, :, 1::2] = z.real, z.imag
                else:
                    y[b, h, :, :half], y[b, h, :, half:] = z.real, z.imag
        out.append(y)
    return dict(zip(("dQ", "dK") if back else ("Q", "K"), out))
