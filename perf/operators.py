"""The gated delta rule, rotary positions with several axes and the
channels-last group norm: the calls that their performance is measured on.

Each case is one call as a vision block with a matrix-state token mixer makes
it: a group norm of the channels-last map ahead of the q, k, v products,
rotary positions (row, column, and time for video) with the L2 norm of the
heads, then the gated delta rule over the tokens (whole maps forward and
backward, single tokens for streams of frames). Map sizes and widths are those
of ``workloads.py``: 56, 28, 14 and 7 pixels a side, a 128 x 512 segmentation
map and a ragged 97 x 101 one, inner widths 192 and 384 in heads of 64, and
heads of 128 where the state is large. Outputs and the workspace are allocated
once, as a training or serving loop keeps them.
"""
from __future__ import annotations

import itertools
import math

import torch

own = False

CHUNK = 64  # tokens that the plain chunked form takes at a time

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # One 7 x 7 map, six heads of 64: the smallest call, where launches count.
        dict(name="delta_fwd_7x7_b1", kind="delta_fwd", batch=1, L=49, packed=0, hk=6, hv=6,
             dk=64, dv=64, dtype="bf16", state=False),
        # A batch of second-stage maps, 384 channels in heads of 64.
        dict(name="delta_fwd_28x28_b32", kind="delta_fwd", batch=32, L=784, packed=0, hk=6, hv=6,
             dk=64, dv=64, dtype="bf16", state=False),
        # Two segmentation maps of 128 x 512 tokens, two value heads to a key
        # head, states of 128 x 128 carried in and out.
        dict(name="delta_fwd_128x512_b2", kind="delta_fwd", batch=2, L=65536, packed=0, hk=2,
             hv=4, dk=128, dv=128, dtype="bf16", state=True),
        # Maps of several sizes packed behind each other (an empty one and one
        # of a single token among them), fp32, heads of 48 and 80.
        dict(name="delta_fwd_packed_f32", kind="delta_fwd", batch=1, L=16000, packed=12, hk=3,
             hv=6, dk=48, dv=80, dtype="f32", state=True),
        # Training on first-stage maps, 192 channels in heads of 64.
        dict(name="delta_bwd_56x56_b32", kind="delta_bwd", batch=32, L=3136, packed=0, hk=3,
             hv=3, dk=64, dv=64, dtype="bf16", state=False),
        # Training on ragged maps in fp32, shared key heads, with states.
        dict(name="delta_bwd_97x101_b2_f32", kind="delta_bwd", batch=2, L=9797, packed=0, hk=2,
             hv=4, dk=32, dv=64, dtype="f32", state=True),
        # Single tokens of 256 streams, 128 x 128 states: the states are read
        # and written once.
        dict(name="delta_step_b256", kind="delta_step", batch=256, T=1, hk=8, hv=16, dk=128,
             dv=128, dtype="bf16"),
        # One stream, four tokens at a time.
        dict(name="delta_step_b1_t4", kind="delta_step", batch=1, T=4, hk=6, hv=6, dk=64, dv=64,
             dtype="f32"),
        # Video: 16 frames of 28 x 28 tokens, three axes, shared key heads.
        dict(name="rotary_fwd_video_b2", kind="rotary_fwd", batch=2, grid_t=16, grid_h=28,
             grid_w=28, hq=12, hk=4, dim=128, pairs=60, interleaved=False, norm=False,
             dtype="bf16"),
        # Training on first-stage maps: two axes, with the norm.
        dict(name="rotary_bwd_56x56_b32", kind="rotary_bwd", batch=32, grid_t=0, grid_h=56,
             grid_w=56, hq=3, hk=3, dim=64, pairs=32, interleaved=True, norm=True, dtype="f32"),
        # The norm of a batch of first-stage maps, 32 groups of six channels.
        dict(name="gnorm_fwd_56x56_b32", kind="gnorm_fwd", batch=32, P=3136, channels=192,
             groups=32, act="silu", dtype="bf16"),
        # Training on the segmentation maps.
        dict(name="gnorm_bwd_128x512_b2", kind="gnorm_bwd", batch=2, P=65536, channels=192,
             groups=8, act="silu", dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["delta_fwd", "delta_fwd", "delta_bwd", "delta_bwd", "delta_step",
                       "rotary_fwd", "rotary_bwd", "gnorm_fwd", "gnorm_bwd"])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]))
    if kind.startswith("delta"):
        hk = rng.choice([1, 2, 3, 4, 6, 8])
        hv = hk * rng.choice([1, 1, 2, 3])
        dk, dv = rng.choice([32, 48, 64, 64, 96, 128]), rng.choice([32, 64, 64, 80, 128])
        if kind == "delta_step":
            batch = _log(rng, 1, 256)
            while batch * hv * dk * dv > 256 * 16 * 128 * 128:
                batch //= 2
            return dict(c, batch=batch, T=rng.choice([1, 1, 1, 2, 5]), hk=hk, hv=hv, dk=dk, dv=dv)
        L, batch, packed = _log(rng, 1, 20000), _log(rng, 1, 32), 0
        if rng.random() < 0.25:
            batch, packed, L = 1, rng.choice([3, 5, 9, 17]), max(L, 40)
        # token and head count times the state's size: at most a quarter of
        # the largest forward case
        most = 2 * 65536 * 4 * 128 * 128 // (4 if kind == "delta_fwd" else 8)
        while batch * L * hv * dk * dv > most and batch > 1:
            batch = max(1, batch * 2 // 3)
        while batch * L * hv * dk * dv > most:
            L = max(1, L * 2 // 3)
        return dict(c, batch=batch, L=L, packed=packed, hk=hk, hv=hv, dk=dk, dv=dv,
                    state=rng.random() < 0.4)
    if kind.startswith("rotary"):
        grid_t = rng.choice([0, 0, _log(rng, 2, 24)])
        grid_h, grid_w = _log(rng, 1, 97), _log(rng, 1, 101)
        hq = rng.choice([1, 2, 3, 6, 8, 12])
        hk = rng.choice([h for h in (1, 2, 3, 4, 6) if h <= hq])
        dim = rng.choice([32, 48, 64, 64, 80, 128])
        axes = 3 if grid_t else 2
        pairs = dim // 2 if rng.random() < 0.6 else rng.randint(axes, dim // 2)
        batch = _log(rng, 1, 32)
        while batch * max(1, grid_t) * grid_h * grid_w * (hq + hk) * dim > 32 * 3136 * 6 * 64:
            if batch > 1:
                batch //= 2
            else:
                grid_h = max(1, grid_h // 2)
        return dict(c, batch=batch, grid_t=grid_t, grid_h=grid_h, grid_w=grid_w, hq=hq, hk=hk,
                    dim=dim, pairs=pairs, interleaved=rng.random() < 0.5,
                    norm=rng.random() < 0.5)
    groups = rng.choice([1, 3, 4, 8, 16, 32])
    channels = groups * _log(rng, 1, max(2, 1536 // groups))
    batch, P = _log(rng, 1, 128), _log(rng, 1, 65536)
    while batch * P * channels > 2 * 65536 * 192:
        if batch > 1:
            batch //= 2
        else:
            P //= 2
    return dict(c, batch=batch, P=P, channels=channels, groups=groups,
                act=rng.choice(["silu", "silu", "none"]))


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """Tokens of each sequence of a packed case: uneven cuts of L, with an
    empty sequence and one of a single token among them."""
    n, L = case["packed"], case["L"]
    weight = [0.0, 0.0] + [1.0 + 3.0 * ((7 * i) % 5) for i in range(n - 2)]
    left = L - 1
    got = [int(left * w / sum(weight)) for w in weight]
    got[1] = 1
    got[-1] += L - sum(got)
    return got[2:3] + got[0:2] + got[3:]


def _delta_inputs(case, seed):
    """Keys and queries of unit length that share a direction within a head
    (neighbouring pixels are alike), log decays -A softplus(.) of a Mamba
    initialisation, write strengths of a sigmoid."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _TORCH[case["dtype"]]
    B, L = case["batch"], case.get("L", case.get("T"))
    hk, hv, dk, dv = case["hk"], case["hv"], case["dk"], case["dv"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def unit(x):
        return (x / x.square().sum(-1, keepdim=True).sqrt()).to(dt)

    s = dict(q=unit(normal(B, L, hk, dk) + normal(B, 1, hk, dk)),
             k=unit(normal(B, L, hk, dk) + normal(B, 1, hk, dk)),
             v=normal(B, L, hv, dv).to(dt))
    step = torch.exp(torch.rand(hv, generator=g, device="cuda") * math.log(100.0) + math.log(1e-3))
    A = 1.0 + 15.0 * torch.rand(hv, generator=g, device="cuda")
    raw = 0.5 * normal(B, L, hv) + torch.log(torch.expm1(step))
    s["g"] = -A * torch.log1p(torch.exp(raw))
    s["beta"] = torch.sigmoid(normal(B, L, hv))
    s["scale"] = dk ** -0.5
    n = case.get("packed") or B
    s["cu"] = None
    if case.get("packed"):
        lengths = _lengths(case)
        s["cu"] = torch.tensor([0, *itertools.accumulate(lengths)], dtype=torch.int32,
                               device="cuda")
        s["longest"] = max(lengths)
    if case["kind"] == "delta_step":
        # more states than rows, taken in an order of the server's
        s["pool"] = 0.3 * normal(B + 3, hv, dk, dv)
        s["slots"] = torch.randperm(B + 3, generator=g, device="cuda")[:B].to(torch.int32)
        s["o"] = torch.empty_like(s["v"])
        return s
    s["h0"] = 0.3 * normal(n, hv, dk, dv) if case["state"] else None
    if case["kind"] == "delta_fwd":
        s["o"] = torch.empty_like(s["v"])
        s["hT"] = torch.empty_like(s["h0"]) if case["state"] else None
    else:
        s["do"] = normal(B, L, hv, dv).to(dt)
        s["dhT"] = 0.3 * normal(n, hv, dk, dv) if case["state"] else None
        s["dh0"] = torch.empty_like(s["h0"]) if case["state"] else None
        for name in ("q", "k", "v", "g", "beta"):
            s["d" + name] = torch.empty_like(s[name])
    return s


def _rotary_inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _TORCH[case["dtype"]]
    T, H, W = case["grid_t"], case["grid_h"], case["grid_w"]
    sides = ([T] if T else []) + [H, W]
    B, L, D = case["batch"], math.prod(sides), case["dim"]
    hq, hk, pairs = case["hq"], case["hk"], case["pairs"]
    s = dict(pos=torch.cartesian_prod(*[torch.arange(n, device="cuda") for n in sides])
             .reshape(1, L, len(sides)).to(torch.int32).contiguous())
    # the axes share the pairs as evenly as they go, each with its own
    # frequencies of base 10000
    cut = [pairs * i // len(sides) for i in range(len(sides) + 1)]
    s["sections"] = [b - a for a, b in zip(cut, cut[1:])]
    s["inv_freq"] = torch.cat([10000.0 ** (-torch.arange(n, device="cuda") / max(n, 1))
                               for n in s["sections"]]).float()
    # queries, keys and values come from one product: views of its output
    qkv = torch.randn(B, L, (hq + 2 * hk) * D, generator=g, device="cuda").to(dt)
    s["q"] = qkv[..., :hq * D].unflatten(-1, (hq, D))
    s["k"] = qkv[..., hq * D:(hq + hk) * D].unflatten(-1, (hk, D))
    names = ("yq", "yk") if case["kind"] == "rotary_fwd" else ("dxq", "dxk")
    for name, h in zip(names, (hq, hk)):
        s[name] = torch.empty(B, L, h, D, dtype=dt, device="cuda")
    if case["kind"] == "rotary_bwd":
        s["dq"] = torch.randn(B, L, hq, D, generator=g, device="cuda").to(dt)
        s["dk"] = torch.randn(B, L, hk, D, generator=g, device="cuda").to(dt)
    s.update(interleaved=case["interleaved"], eps=1e-6 if case["norm"] else None)
    return s


def _gnorm_inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _TORCH[case["dtype"]]
    N, P, C, G = case["batch"], case["P"], case["channels"], case["groups"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = dict(x=(normal(N, P, C) + 0.5 + 0.5 * normal(1, 1, C)).to(dt), gamma=1 + 0.1 * normal(C),
             beta=0.1 * normal(C), groups=G, eps=1e-5, act=case["act"])
    if case["kind"] == "gnorm_fwd":
        s["y"] = torch.empty_like(s["x"])
        s["mean"], s["rstd"] = torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
    else:
        x = s["x"].double().view(N, P, G, C // G)
        mean = x.mean((1, 3))
        var = (x - mean.view(N, 1, G, 1)).square().mean((1, 3))
        s["mean"], s["rstd"] = mean.float(), (1 / torch.sqrt(var + s["eps"])).float()
        s["dy"] = normal(N, P, C).to(dt)
        s["dx"] = torch.empty_like(s["x"])
        s["dgamma"], s["dbeta"] = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    return s


def prepare(case, seed):
    make = {"d": _delta_inputs, "r": _rotary_inputs, "g": _gnorm_inputs}[case["kind"][0]]
    return dict(make(case, seed), kind=case["kind"])


# --------------------------------------------------------------- plain forms

def _to_batch(x, s, fill=0.0):
    """Packed tokens [1, L, ...] as one row a sequence [n, longest, ...]."""
    if s["cu"] is None:
        return x
    cu = s["cu"].long()
    at = cu[:-1, None] + torch.arange(s["longest"], device="cuda")
    held = at < cu[1:, None]
    y = x[0][at.clamp(max=x.shape[1] - 1)]
    return torch.where(held.view(*held.shape, *[1] * (x.dim() - 2)), y, fill)


def _from_batch(y, s, L):
    """The inverse: rows of sequences back to packed tokens."""
    if s["cu"] is None:
        return y
    cu = s["cu"].long()
    at = torch.arange(L, device="cuda")
    row = (at[:, None] >= cu[None, 1:]).sum(1)
    return y[row, at - cu[row]][None]


def _in_chunks(x):
    """[B, L, H, d] -> [B, H, chunks, CHUNK, d], zeros behind the end."""
    B, L, H, d = x.shape
    n = -(-L // CHUNK)
    x = torch.cat([x, x.new_zeros(B, n * CHUNK - L, H, d)], 1)
    return x.view(B, n, CHUNK, H, d).permute(0, 3, 1, 2, 4).contiguous()


def _unit_lower_inverse(X):
    """(I + X)^-1 of strictly lower triangular X [..., CHUNK, CHUNK]: blocks of
    1, 2, 4, ... on the diagonal, joined in pairs."""
    lead = X.shape[:-2]
    T = X.new_ones(*lead, CHUNK, 1, 1)
    size = 1
    while size < CHUNK:
        n = CHUNK // (2 * size)
        blocks = X.view(*lead, n, 2, size, n, 2, size)[..., :, 1, :, :, 0, :]
        low = torch.diagonal(blocks, dim1=-4, dim2=-2).movedim(-1, -3)
        a, b = T.view(*lead, n, 2, size, size).unbind(-3)
        low = -(b.contiguous() @ (low.contiguous() @ a.contiguous()))
        T = torch.cat([torch.cat([a, torch.zeros_like(a)], -1), torch.cat([low, b], -1)], -2)
        size *= 2
    return T.view(*lead, CHUNK, CHUNK)


def _delta_plain(q, k, v, g, beta, h0, scale):
    """The chunked form in fp32 on [B, L, H, d]: o and the last state."""
    B, L, hv = g.shape
    heads = hv // q.shape[2]
    q, k = (_in_chunks(x.repeat_interleave(heads, 2)) for x in (q, k))
    v, g, beta = _in_chunks(v), _in_chunks(g[..., None])[..., 0], _in_chunks(beta[..., None])
    beta = beta.transpose(-1, -2)
    G = g.cumsum(-1)
    low = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda").tril()
    D = torch.exp(torch.where(low, G[..., :, None] - G[..., None, :], -math.inf))
    kt = k.transpose(-1, -2).contiguous()
    T = _unit_lower_inverse(((k @ kt) * D).tril(-1) * beta)
    P = (q @ kt) * D * (beta * scale)
    eG = torch.exp(G)[..., None]
    E0, W = T @ v, T @ (k * eG)
    qe = q * (eG * scale)
    last = torch.exp(G[..., -1:])[..., None]
    kd = (kt * (beta * torch.exp(G[..., -1:] - G)[..., None, :])).contiguous()
    S = v.new_zeros(B, hv, k.shape[-1], v.shape[-1]) if h0 is None else h0
    o = []
    for n in range(v.shape[2]):
        E = E0[:, :, n] - W[:, :, n] @ S
        o.append(qe[:, :, n] @ S + P[:, :, n] @ E)
        S = last[:, :, n] * S + kd[:, :, n] @ E
    o = torch.stack(o, 2).permute(0, 2, 3, 1, 4).reshape(B, -1, hv, v.shape[-1])[:, :L]
    return o, S


def _delta_fwd_plain(s):
    x = [_to_batch(s[n], s).float() for n in ("q", "k", "v", "g", "beta")]
    o, S = _delta_plain(*x, s["h0"], s["scale"])
    out = dict(o=_from_batch(o, s, s["v"].shape[1]).to(s["v"].dtype))
    return dict(out, hT=S) if s["h0"] is not None else out


def _delta_bwd_plain(s):
    names = ("q", "k", "v", "g", "beta")
    x = [s[n].float().requires_grad_() for n in names]
    h0 = None if s["h0"] is None else s["h0"].clone().requires_grad_()
    with torch.enable_grad():
        o, S = _delta_plain(*[_to_batch(t, s) for t in x], h0, s["scale"])
        o = _from_batch(o, s, s["v"].shape[1])
        ends, seeds = ([o], [s["do"].float()]) if h0 is None else ([o, S],
                                                                   [s["do"].float(), s["dhT"]])
        grads = torch.autograd.grad(ends, x if h0 is None else x + [h0], seeds)
    out = {"d" + n: t.to(s[n].dtype) for n, t in zip(names, grads)}
    return out if h0 is None else dict(out, dh0=grads[-1])


def _delta_step_plain(s):
    heads = s["v"].shape[2] // s["q"].shape[2]
    q, k = (s[n].float().repeat_interleave(heads, 2) for n in ("q", "k"))
    v, at = s["v"].float(), s["slots"].long()
    S, o = s["pool"][at], []
    for t in range(v.shape[1]):
        S = S * torch.exp(s["g"][:, t])[..., None, None]
        e = v[:, t] - (S * k[:, t, ..., None]).sum(-2)
        S = S + k[:, t, ..., None] * (s["beta"][:, t, :, None] * e)[..., None, :]
        o.append((S * q[:, t, ..., None]).sum(-2) * s["scale"])
    s["pool"][at] = S
    return dict(o=torch.stack(o, 1).to(s["v"].dtype), pool=s["pool"])


def _turn(x, cos, sin, interleaved):
    n = cos.shape[-1]
    if interleaved:
        a, b, rest = x[..., 0:2 * n:2], x[..., 1:2 * n:2], x[..., 2 * n:]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2),
                          rest], -1)
    a, b, rest = x[..., :n], x[..., n:2 * n], x[..., 2 * n:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], -1)


def _angles(s, kind):
    """[1, L, 1, pairs]: each pair's axis position times its frequency."""
    axis = torch.cat([torch.full((n,), i, device="cuda") for i, n in enumerate(s["sections"])])
    return (s["pos"].to(kind)[..., axis] * s["inv_freq"].to(kind))[:, :, None]


def _rotary_fwd_plain(s):
    a = _angles(s, torch.float32)
    out = {}
    for name, y in (("q", "yq"), ("k", "yk")):
        x = s[name].float()
        if s["eps"] is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) + s["eps"])
        out[y] = _turn(x, torch.cos(a), torch.sin(a), s["interleaved"]).to(s[name].dtype)
    return out


def _rotary_bwd_plain(s):
    a = _angles(s, torch.float32)
    out = {}
    for name, dx in (("q", "dxq"), ("k", "dxk")):
        d = _turn(s["d" + name].float(), torch.cos(a), -torch.sin(a), s["interleaved"])
        if s["eps"] is not None:
            x = s[name].float()
            r = 1 / torch.sqrt(x.square().sum(-1, keepdim=True) + s["eps"])
            d = r * (d - x * ((x * d).sum(-1, keepdim=True) * r * r))
        out[dx] = d.to(s[name].dtype)
    return out


def _gnorm_parts(s):
    x = s["x"].float()
    N, P, C = x.shape
    G = s["groups"]
    return x.view(N, P, G, C // G), s["gamma"].view(G, C // G), s["beta"].view(G, C // G)


def _gnorm_fwd_plain(s):
    x, gamma, beta = _gnorm_parts(s)
    mean = x.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean((1, 3), keepdim=True) + s["eps"])
    z = (x - mean) * rstd * gamma + beta
    y = z / (1 + torch.exp(-z)) if s["act"] == "silu" else z
    return dict(y=y.reshape(s["x"].shape).to(s["x"].dtype), mean=mean[:, 0, :, 0],
                rstd=rstd[:, 0, :, 0])


def _gnorm_bwd_plain(s):
    x, gamma, beta = _gnorm_parts(s)
    rstd = s["rstd"][:, None, :, None]
    xh = (x - s["mean"][:, None, :, None]) * rstd
    dz = s["dy"].float().view(x.shape)
    if s["act"] == "silu":
        z = xh * gamma + beta
        sig = 1 / (1 + torch.exp(-z))
        dz = dz * (sig * (1 + z * (1 - sig)))
    dgamma, dbeta = (dz * xh).sum((0, 1)).flatten(), dz.sum((0, 1)).flatten()
    dh = dz * gamma
    dx = rstd * (dh - dh.mean((1, 3), keepdim=True) - xh * (dh * xh).mean((1, 3), keepdim=True))
    return dict(dx=dx.reshape(s["x"].shape).to(s["x"].dtype), dgamma=dgamma, dbeta=dbeta)


_PLAIN = dict(delta_fwd=_delta_fwd_plain, delta_bwd=_delta_bwd_plain,
              delta_step=_delta_step_plain, rotary_fwd=_rotary_fwd_plain,
              rotary_bwd=_rotary_bwd_plain, gnorm_fwd=_gnorm_fwd_plain,
              gnorm_bwd=_gnorm_bwd_plain)


# ------------------------------------------------------------- the library's

def _workspace(s, nbytes):
    """Kept with the state, as a program keeps it between its calls."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(nbytes(), 16), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _run_own(s):
    from paper_2412_16602_amd import vmb
    kind = s["kind"]
    if kind in ("delta_fwd", "delta_bwd"):
        B, L, hk, dk = s["q"].shape
        hv, dv = s["v"].shape[2:]
        n = B if s["cu"] is None else s["cu"].numel() - 1
        ws = _workspace(s, lambda: vmb.vmb_gated_delta_workspace_bytes(
            kind == "delta_bwd", B, L, n, hk, hv, dk, dv, s["q"].dtype))
        args = (s["q"], s["k"], s["v"], s["g"], s["beta"])
        more = dict(scale=s["scale"], h0=s["h0"], cu_seqlens=s["cu"], workspace=ws)
        if kind == "delta_fwd":
            vmb.vmb_gated_delta_fwd(*args, s["o"], hT=s["hT"], **more)
            return dict(o=s["o"]) if s["hT"] is None else dict(o=s["o"], hT=s["hT"])
        vmb.vmb_gated_delta_bwd(*args, s["do"], s["dq"], s["dk"], s["dv"], s["dg"], s["dbeta"],
                                dhT=s["dhT"], dh0=s["dh0"], **more)
        out = {n: s[n] for n in ("dq", "dk", "dv", "dg", "dbeta")}
        return out if s["dh0"] is None else dict(out, dh0=s["dh0"])
    if kind == "delta_step":
        vmb.vmb_gated_delta_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["pool"], s["o"],
                                 slots=s["slots"], scale=s["scale"])
        return dict(o=s["o"], pool=s["pool"])
    if kind == "rotary_fwd":
        vmb.vmb_axis_rotary_fwd(s["q"], s["k"], s["pos"], s["inv_freq"], s["sections"], s["yq"],
                                s["yk"], interleaved=s["interleaved"], norm_eps=s["eps"])
        return dict(yq=s["yq"], yk=s["yk"])
    if kind == "rotary_bwd":
        q, k = (s["q"], s["k"]) if s["eps"] is not None else (None, None)
        vmb.vmb_axis_rotary_bwd(s["dq"], s["dk"], q, k, s["pos"], s["inv_freq"], s["sections"],
                                s["dxq"], s["dxk"], interleaved=s["interleaved"],
                                norm_eps=s["eps"])
        return dict(dxq=s["dxq"], dxk=s["dxk"])
    N, P, C = s["x"].shape
    act = vmb.VMB_ACT_SILU if s["act"] == "silu" else vmb.VMB_ACT_NONE
    ws = _workspace(s, lambda: vmb.vmb_group_norm_act_workspace_bytes(
        kind == "gnorm_bwd", N, P, C, s["groups"]))
    if kind == "gnorm_fwd":
        vmb.vmb_group_norm_act_fwd(s["x"], s["gamma"], s["beta"], s["groups"], s["eps"], act,
                                   s["y"], s["mean"], s["rstd"], workspace=ws)
        return dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
    vmb.vmb_group_norm_act_bwd(s["dy"], s["x"], s["gamma"], s["beta"], s["mean"], s["rstd"],
                               s["groups"], act, s["dx"], s["dgamma"], s["dbeta"], workspace=ws)
    return dict(dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])


def run(state):
    return _run_own(state) if own else _PLAIN[state["kind"]](state)


# ------------------------------------------------------------------- in 64 bits

def _delta_walk(q, k, v, g, beta, S, scale, keep=None):
    """The recurrence token by token in 64 bits on [B, L, H, d]."""
    o, e = torch.empty_like(v), torch.empty_like(v)
    for t in range(v.shape[1]):
        if keep is not None:
            keep.append(S)
        S = S * torch.exp(g[:, t])[..., None, None]
        e[:, t] = v[:, t] - (S * k[:, t, ..., None]).sum(-2)
        S = S + (beta[:, t, :, None] * k[:, t])[..., None] * e[:, t, :, None]
        o[:, t] = scale * (S * q[:, t, ..., None]).sum(-2)
    return o, e, S


def _delta_walk_back(q, k, v, g, beta, S0, scale, do, dS):
    """Its gradients, walking back over the states before each token."""
    states = []
    _, e, last = _delta_walk(q, k, v, g, beta, S0, scale, states)
    states.append(last)
    dq, dk, dv, dg, db = (torch.empty_like(x) for x in (q, k, v, g, beta))
    for t in reversed(range(v.shape[1])):
        kt, b = k[:, t], beta[:, t, :, None]
        dq[:, t] = scale * (states[t + 1] * do[:, t, :, None]).sum(-1)
        dS = dS + scale * q[:, t, ..., None] * do[:, t, :, None]
        # S_t = S' + k (b e)^T with S' = a S_{t-1} and e = v - S'^T k
        du = (dS * kt[..., None]).sum(-2)
        db[:, t] = (du * e[:, t]).sum(-1)
        de = b * du
        dv[:, t] = de
        a = torch.exp(g[:, t])[..., None, None]
        Sp = a * states[t]
        dk[:, t] = (dS * (b * e[:, t])[..., None, :]).sum(-1) - (Sp * de[..., None, :]).sum(-1)
        dS = dS - kt[..., None] * de[..., None, :]
        dg[:, t] = (dS * Sp).sum((-1, -2))
        dS = a * dS
    return dq, dk, dv, dg, db, dS


def _delta_exact(case, s):
    f = torch.float64
    heads = case["hv"] // case["hk"]
    x = [s[n].to(f) for n in ("q", "k", "v", "g", "beta")]
    x[0], x[1] = (t.repeat_interleave(heads, 2) for t in x[:2])

    def fold(t):  # sum over the value heads that share a key head
        return t.unflatten(2, (case["hk"], heads)).sum(3)

    if case["kind"] == "delta_step":
        pool = s["pool"].to(f)
        at = s["slots"].long()
        o, _, S = _delta_walk(*x, pool[at], s["scale"])
        pool[at] = S
        return dict(o=o, pool=pool)
    size = case["batch"] * case["hv"] * case["dk"] * case["dv"]
    longest = s.get("longest", case["L"])
    steps = case["L"]
    back = case["kind"] == "delta_bwd"
    # about 0.1 ms a token forward and 0.25 backward, and the time of the
    # states' own traffic; backward keeps a state a token
    if steps * (1e-4 + size * 8e-11) * (2.5 if back else 1) > 14:
        return None
    if back and longest * size * 8 > 60e9:
        return None
    ends = [0, case["L"]] if s["cu"] is None else s["cu"].tolist()
    outs = []
    for i, (a, b) in enumerate(zip(ends, ends[1:])):
        rows = slice(None) if s["cu"] is None else slice(i, i + 1)
        part = [t[:, a:b].contiguous() for t in x]
        zero = x[2].new_zeros(case["batch"], case["hv"], case["dk"], case["dv"])
        S0 = zero if s["h0"] is None else s["h0"][rows].to(f)
        if back:
            dS = zero if s["dhT"] is None else s["dhT"][rows].to(f)
            outs.append(_delta_walk_back(*part, S0, s["scale"], s["do"][:, a:b].to(f), dS))
        else:
            o, _, S = _delta_walk(*part, S0, s["scale"])
            outs.append((o, S))
    *tokens, S = zip(*outs)
    tokens, S = [torch.cat(t, 1) for t in tokens], torch.cat(S, 0)
    if not back:
        return dict(o=tokens[0], hT=S) if case["state"] else dict(o=tokens[0])
    out = dict(zip(("dq", "dk", "dv", "dg", "dbeta"),
                   [fold(tokens[0]), fold(tokens[1]), *tokens[2:]]))
    return dict(out, dh0=S) if case["state"] else out


def _rotary_exact(s):
    """By complex numbers: a pair times e^(i theta), or its conjugate."""
    spin = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       _angles(s, torch.float64))
    back = s["kind"] == "rotary_bwd"
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        d = s["d" + name].double() if back else x
        r = 1.0
        if s["eps"] is not None:
            r = (x.square().sum(-1, keepdim=True) + s["eps"]).rsqrt()
        n = spin.shape[-1]
        pair = d[..., :2 * n]
        pair = pair.unflatten(-1, (n, 2)) if s["interleaved"] else pair.unflatten(
            -1, (2, n)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous())
                               * (spin.conj() if back else spin))
        z = (z if s["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        z = torch.cat([z, d[..., 2 * n:]], -1)
        if back and s["eps"] is not None:
            z = z - x * (x * z).sum(-1, keepdim=True) * r * r
        out[("dx" if back else "y") + name] = z * r
    return out


def _gnorm_exact(s):
    N, P, C = s["x"].shape
    G = s["groups"]
    # groups ahead: [N, G, P * C / G]
    x = s["x"].double().view(N, P, G, -1).transpose(1, 2)
    w = s["gamma"].double().view(1, G, 1, -1)
    b = s["beta"].double().view(1, G, 1, -1)
    if s["kind"] == "gnorm_fwd":
        mean = x.flatten(2).mean(-1)
        rstd = (x.flatten(2).var(-1, unbiased=False) + s["eps"]).rsqrt()
        z = (x - mean[..., None, None]) * rstd[..., None, None] * w + b
        y = z * torch.sigmoid(z) if s["act"] == "silu" else z
        return dict(y=y.transpose(1, 2).reshape(N, P, C), mean=mean, rstd=rstd)
    mean, rstd = (s[n].double()[..., None, None] for n in ("mean", "rstd"))
    xh = (x - mean) * rstd
    d = s["dy"].double().view(N, P, G, -1).transpose(1, 2)
    if s["act"] == "silu":
        z = xh * w + b
        d = d * torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    dgamma, dbeta = (d * xh).sum((0, 2)).flatten(), d.sum((0, 2)).flatten()
    m = x.shape[2] * x.shape[3]
    s1, s2 = ((d * w * t).sum((2, 3), keepdim=True) / m for t in (torch.ones_like(xh), xh))
    dx = rstd * (d * w - s1 - xh * s2)
    return dict(dx=dx.transpose(1, 2).reshape(N, P, C), dgamma=dgamma, dbeta=dbeta)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("delta"):
        return _delta_exact(case, s)
    return _rotary_exact(s) if case["kind"].startswith("rotary") else _gnorm_exact(s)


# ------------------------------------------------------------------------ work

def work(case):
    """Bytes: inputs read once and outputs written once. Operations: the
    recurrence's own (6 dk dv a token and head forward and in a step, 16
    backward with the states recomputed), or a few a value."""
    e = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    if kind.startswith("delta"):
        hk, hv, dk, dv = case["hk"], case["hv"], case["dk"], case["dv"]
        tokens = case["batch"] * case.get("L", case.get("T"))
        state = case["batch"] if not case.get("packed") else case["packed"]
        state *= hv * dk * dv * 4
        qkv = tokens * (2 * hk * dk + hv * dv) * e + tokens * hv * 8
        o = tokens * hv * dv * e
        f = tokens * hv * dk * dv
        if kind == "delta_step":
            return {"bytes": qkv + o + 2 * state, "flops": 6 * f}
        held = 2 * state if case["state"] else 0
        if kind == "delta_fwd":
            return {"bytes": qkv + o + held, "flops": 6 * f}
        return {"bytes": 2 * qkv + o + (3 * state if case["state"] else 0), "flops": 16 * f}
    if kind.startswith("rotary"):
        L = max(1, case["grid_t"]) * case["grid_h"] * case["grid_w"]
        n = case["batch"] * L * (case["hq"] + case["hk"]) * case["dim"]
        reads = 2 if kind == "rotary_bwd" and case["norm"] else 1
        return {"bytes": n * e * (reads + 1) + L * 4 * (3 if case["grid_t"] else 2),
                "flops": 6 * n}
    n = case["batch"] * case["P"] * case["channels"]
    return {"bytes": n * e * (2 if kind == "gnorm_fwd" else 3), "flops": 12 * n}
