"""64-bit references of the gated delta rule, the rotary positions and the
channels-last group norm, from their definitions (numpy, token by token), and
the comparisons that the tests of those operators share."""
from __future__ import annotations

import numpy as np
import torch

# Bounds on |got - ref|. float32 results, in the 2-norm over the 2-norm of ref:
# 2^-24 a rounding; the longest chains here add some hundreds of terms with
# random signs (a factor of about 20) and the state feeds back through some
# tens of chunks, so 5e-6 leaves a factor of four; a single value may be 40
# times that off, against max(rms, |ref|). bfloat16 results: one rounding, at
# most 2^-8 |ref| a value (half of the spacing at a significand of 1), and
# operands of 16 bits or more inside, 5e-4 of the rms for a single value;
# over a thousand values or more the roundings average 2^-8 / sqrt(3) / 1.4 =
# 1.6e-3, bounded by 2.2e-3.
NORM = {torch.float32: 5e-6, torch.bfloat16: 2.2e-3}
INNER = 5e-4


def check(got: torch.Tensor, ref: np.ndarray, what: str, kind=None):
    kind = got.dtype if kind is None else kind
    x = got.detach().double().cpu().numpy()
    assert x.shape == ref.shape, (what, x.shape, ref.shape)
    assert np.all(np.isfinite(x)), f"{what}: values that are not finite"
    if not ref.size:
        return
    d, norm = np.abs(x - ref), np.linalg.norm(ref)
    rms = norm / np.sqrt(ref.size)
    if rms == 0:
        assert not d.any(), f"{what}: not zero"
        return
    rel = np.linalg.norm(d) / norm
    if kind == torch.bfloat16:
        big = np.max((d - 2.0**-8 * np.abs(ref)) / rms)
        most = INNER
        norm_most = NORM[kind] if ref.size >= 1000 else 2.0**-8 + INNER
    else:
        big = np.max(d / np.maximum(np.abs(ref), rms))
        most, norm_most = 40 * NORM[kind], NORM[kind]
    print(f"{what}: rel {rel:.2e} (at most {norm_most:.1e}), largest {big:.2e}", flush=True)
    assert rel <= norm_most, f"{what}: relative error {rel:.3e} > {norm_most}"
    assert big <= most, f"{what}: largest error {big:.3e} > {most}"


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def per_value_head(x, heads_v):
    return np.repeat(x, heads_v // x.shape[2], axis=2)


def delta_walk(q, k, v, g, beta, scale, h0=None, keep=False):
    """q, k, v [B, L, H, d] (q, k already per value head): o, last state, and
    with keep the states before each token (the last behind) and the errors."""
    B, L, H, dv = v.shape
    S = np.zeros((B, H, q.shape[-1], dv)) if h0 is None else h0.copy()
    o, e, states = np.empty_like(v), np.empty_like(v), []
    for t in range(L):
        if keep:
            states.append(S)
        S = S * np.exp(g[:, t])[..., None, None]
        e[:, t] = v[:, t] - np.einsum("bhkv,bhk->bhv", S, k[:, t])
        S = S + (beta[:, t, :, None] * k[:, t])[..., None] * e[:, t, :, None]
        o[:, t] = scale * np.einsum("bhkv,bhk->bhv", S, q[:, t])
    return (o, S, states + [S], e) if keep else (o, S)


def delta_walk_back(q, k, v, g, beta, scale, h0, do, dhT):
    _, _, states, e = delta_walk(q, k, v, g, beta, scale, h0, keep=True)
    dS = np.zeros_like(states[0]) if dhT is None else dhT.copy()
    dq, dk, dv = np.empty_like(q), np.empty_like(k), np.empty_like(v)
    dg, db = np.empty_like(g), np.empty_like(beta)
    for t in reversed(range(v.shape[1])):
        dq[:, t] = scale * np.einsum("bhkv,bhv->bhk", states[t + 1], do[:, t])
        dS = dS + scale * q[:, t][..., None] * do[:, t][..., None, :]
        du = np.einsum("bhkv,bhk->bhv", dS, k[:, t])
        db[:, t] = (du * e[:, t]).sum(-1)
        de = beta[:, t][..., None] * du
        dv[:, t] = de
        decay = np.exp(g[:, t])[..., None, None]
        Sp = decay * states[t]
        dk[:, t] = (np.einsum("bhkv,bhv->bhk", dS, beta[:, t][..., None] * e[:, t])
                    - np.einsum("bhkv,bhv->bhk", Sp, de))
        dS = dS - k[:, t][..., None] * de[..., None, :]
        dg[:, t] = (dS * Sp).sum((-1, -2))
        dS = decay * dS
    return dq, dk, dv, dg, db, dS


def delta_ref(q, k, v, g, beta, scale, h0=None, cu=None, do=None, dhT=None):
    """The forward result (o, hT), or with do the gradients (dq, dk, dv, dg,
    dbeta, dh0), of tensors as the library takes them."""
    hv, hk = v.shape[2], q.shape[2]
    q, k, v, g, beta, h0, do, dhT = (f64(t) for t in (q, k, v, g, beta, h0, do, dhT))
    q, k = per_value_head(q, hv), per_value_head(k, hv)
    B, L = v.shape[:2]
    spans = [(slice(None), slice(0, L))] if cu is None else [
        (slice(i, i + 1), slice(a, b)) for i, (a, b) in enumerate(zip(cu, cu[1:]))]
    parts = []
    for rows, toks in spans:
        x = [t[:, toks] for t in (q, k, v, g, beta)]
        s0 = None if h0 is None else h0[rows]
        if do is None:
            parts.append(delta_walk(*x, scale, s0))
        else:
            parts.append(delta_walk_back(*x, scale, s0, do[:, toks],
                                         None if dhT is None else dhT[rows]))
    *tokens, S = zip(*parts)
    tokens, S = [np.concatenate(t, 1) for t in tokens], np.concatenate(S, 0)
    if do is not None:
        tokens[:2] = [t.reshape(B, L, hk, hv // hk, -1).sum(3) for t in tokens[:2]]
    return (*tokens, S)


def rotary_ref(x, positions, inv_freq, sections, interleaved, eps, dy=None):
    """y of x, or with dy the gradient of x (numpy float64)."""
    n = sum(sections)
    axis = np.repeat(np.arange(len(sections)), sections)
    theta = (positions[..., axis].astype(np.float64) * inv_freq)[:, :, None]
    c, s = np.cos(theta), np.sin(theta)
    d = x if dy is None else dy
    if dy is not None:
        s = -s
    if interleaved:
        first, second = np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)
    else:
        first, second = np.arange(n), np.arange(n, 2 * n)
    y = d.copy()
    y[..., first] = d[..., first] * c - d[..., second] * s
    y[..., second] = d[..., first] * s + d[..., second] * c
    if eps is None:
        return y
    r = 1 / np.sqrt((x * x).sum(-1, keepdims=True) + eps)
    if dy is None:
        return y * r
    return r * (y - x * (x * y).sum(-1, keepdims=True) * r * r)


def group_norm_ref(x, gamma, beta, groups, eps, silu, dy=None, mean=None, rstd=None):
    """(y, mean, rstd), or with dy (dx, dgamma, dbeta); x [N, P, C] float64."""
    N, P, C = x.shape
    x = x.reshape(N, P, groups, C // groups)
    w = np.ones(C) if gamma is None else gamma
    b = np.zeros(C) if beta is None else beta
    w, b = w.reshape(groups, -1), b.reshape(groups, -1)
    if dy is None:
        mean = x.mean((1, 3))
        rstd = 1 / np.sqrt(((x - mean[:, None, :, None]) ** 2).mean((1, 3)) + eps)
    xh = (x - mean[:, None, :, None]) * rstd[:, None, :, None]
    z = xh * w + b
    with np.errstate(over="ignore"):
        sig = 1 / (1 + np.exp(-z))
    if dy is None:
        return (z * sig if silu else z).reshape(N, P, C), mean, rstd
    d = dy.reshape(x.shape)
    if silu:
        d = d * sig * (1 + z * (1 - sig))
    dgamma, dbeta = (d * xh).sum((0, 1)).ravel(), d.sum((0, 1)).ravel()
    dw = d * w
    dx = rstd[:, None, :, None] * (dw - dw.mean((1, 3), keepdims=True)
                                   - xh * (dw * xh).mean((1, 3), keepdims=True))
    return dx.reshape(N, P, C), dgamma, dbeta
