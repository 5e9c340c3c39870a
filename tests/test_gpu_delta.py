"""The gated delta rule (vmb_gated_delta_fwd / _bwd / _step) against the
recurrence in 64 bits: chunks that are full, partial and single, head sizes on
and off the padded widths, shared key heads, packed sequences with empty ones,
strided inputs, states carried in and out, decays of zero, beta of zero and
one, calls split in two, and the step form against the chunked one."""
import numpy as np
import pytest
import torch

from mixer_ref import check, delta_ref
from paper_2412_16602_amd import vmb

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def make(B, L, hk, hv, dk, dv, dtype, seed=0, n=None, alike=1.0):
    g = torch.Generator().manual_seed(seed)
    def normal(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)
    def unit(x):
        return (x / x.norm(dim=-1, keepdim=True)).to(dtype).cuda()
    q = unit(normal(B, L, hk, dk) + alike * normal(B, 1, hk, dk))
    k = unit(normal(B, L, hk, dk) + alike * normal(B, 1, hk, dk))
    v = normal(B, L, hv, dv).to(dtype).cuda()
    gate = (-0.3 * torch.rand(B, L, hv, generator=g, dtype=torch.float64)
            * torch.rand(hv, generator=g, dtype=torch.float64)).float().cuda()
    beta = torch.sigmoid(normal(B, L, hv)).float().cuda()
    n = B if n is None else n
    h0 = (0.3 * normal(n, hv, dk, dv)).float().cuda()
    return q, k, v, gate, beta, h0


def forward(x, h0=None, cu=None, want_state=True, scale=0.125):
    q, k, v, g, beta = x
    o = torch.full(v.shape, float("nan"), dtype=v.dtype, device="cuda")
    n = q.shape[0] if cu is None else len(cu) - 1
    hT = torch.full((n, v.shape[2], q.shape[3], v.shape[3]), float("nan"),
                    device="cuda") if want_state else None
    c = None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda")
    vmb.vmb_gated_delta_fwd(q, k, v, g, beta, o, scale=scale, h0=h0, hT=hT, cu_seqlens=c)
    torch.cuda.synchronize()
    return o, hT


def backward(x, do, h0=None, dhT=None, cu=None, scale=0.125):
    q, k, v, g, beta = x
    def nan(t):
        return torch.full(t.shape, float("nan"), dtype=t.dtype, device="cuda")
    out = [nan(t) for t in x]
    dh0 = None if h0 is None else nan(h0)
    c = None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda")
    vmb.vmb_gated_delta_bwd(q, k, v, g, beta, do, *out, scale=scale, h0=h0, dhT=dhT, dh0=dh0,
                            cu_seqlens=c)
    torch.cuda.synchronize()
    return out + ([] if dh0 is None else [dh0])


SHAPES = [  # batch, L, key heads, value heads, dk, dv
    (1, 1, 1, 1, 8, 8), (2, 2, 1, 2, 64, 64), (1, 31, 2, 2, 32, 16), (1, 32, 1, 1, 32, 32),
    (2, 33, 1, 3, 48, 80), (1, 63, 2, 4, 64, 64), (3, 64, 1, 1, 128, 128), (1, 65, 2, 2, 96, 40),
    (1, 130, 1, 2, 128, 64), (2, 300, 2, 2, 24, 256), (1, 1000, 1, 2, 64, 128),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward(shape, dtype):
    *x, h0 = make(*shape, dtype)
    for state in (h0, None):
        o, hT = forward(x, state)
        ro, rS = delta_ref(*x, 0.125, state)
        check(o, ro, f"o {shape}")
        check(hT, rS, f"hT {shape}")


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward_bf16_without_states(shape):
    """No float32 output: the operands that are computed hold 16 bits."""
    *x, _ = make(*shape, BF16, seed=3)
    o, _ = forward(x, want_state=False)
    check(o, delta_ref(*x, 0.125)[0], f"o {shape}")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_backward(shape, dtype):
    *x, h0 = make(*shape, dtype, seed=1)
    g = torch.Generator().manual_seed(5)
    do = torch.randn(x[2].shape, generator=g).to(dtype).cuda()
    dhT = torch.randn(h0.shape, generator=g).cuda() * 0.3
    names = ("dq", "dk", "dv", "dg", "dbeta", "dh0")
    for h, d in ((h0, dhT), (None, None)):
        got = backward(x, do, h, d)
        ref = delta_ref(*x, 0.125, h, do=do, dhT=d)
        for name, a, b in zip(names, got, ref):
            check(a, b, f"{name} {shape}")


PACKED = [[0, 1], [0, 0, 5, 5, 6, 70], [0, 64, 128, 129, 129, 400], [0, 200, 201, 201, 264, 265]]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("cu", PACKED, ids=str)
def test_packed(cu, dtype):
    *x, h0 = make(1, cu[-1], 1, 2, 64, 48, dtype, seed=2, n=len(cu) - 1)
    o, hT = forward(x, h0, cu)
    ro, rS = delta_ref(*x, 0.125, h0, cu)
    check(o, ro, "o")
    check(hT, rS, "hT")
    do = torch.randn(x[2].shape, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    got = backward(x, do, h0, h0.flip(0).contiguous(), cu)
    ref = delta_ref(*x, 0.125, h0, cu, do=do, dhT=h0.flip(0))
    for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), got, ref):
        check(a, b, name)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_views_of_one_product(dtype):
    """q, k, v as slices of one [B, L, width] tensor give what copies give."""
    B, L, hk, hv, dk, dv = 2, 77, 2, 4, 32, 48
    *x, h0 = make(B, L, hk, hv, dk, dv, dtype, seed=4)
    wide = torch.cat([t.flatten(2) for t in x[:3]] + [torch.full((B, L, 16), float("nan"),
                     dtype=dtype, device="cuda")], -1)
    q = wide[..., :hk * dk].unflatten(-1, (hk, dk))
    k = wide[..., hk * dk:2 * hk * dk].unflatten(-1, (hk, dk))
    v = wide[..., 2 * hk * dk:2 * hk * dk + hv * dv].unflatten(-1, (hv, dv))
    assert not q.is_contiguous()
    a, b = forward(x, h0), forward([q, k, v] + x[3:], h0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    do = torch.randn(B, L, hv, dv, device="cuda").to(dtype)
    for s, t in zip(backward(x, do, h0), backward([q, k, v] + x[3:], do, h0)):
        assert torch.equal(s, t)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_gates_at_their_ends(dtype):
    """Decays of zero (-inf and below -128) forget all before them, beta of 0
    writes nothing, beta of 1 replaces, decays of exactly 1 keep."""
    *x, h0 = make(1, 150, 1, 4, 64, 32, dtype, seed=6)
    q, k, v, g, beta = x
    g[:, 40, 0], g[:, 100, 0], g[:, 101, 0] = -float("inf"), -200.0, -float("inf")
    g[..., 1], beta[..., 1] = 0.0, 1.0
    beta[:, ::3, 2] = 0.0
    g[..., 3] = -30.0
    do = torch.randn(v.shape, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    o, hT = forward(x, h0)
    ro, rS = delta_ref(*x, 0.125, h0)
    check(o, ro, "o")
    check(hT, rS, "hT")
    got = backward(x, do, h0, h0)
    ref = delta_ref(*x, 0.125, h0, do=do, dhT=h0)
    for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), got, ref):
        check(a, b, name)
    assert not got[3][:, [40, 100, 101], 0].any()


@pytest.mark.parametrize("decay", ["slow", "fast", "gone"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 4200, 1, 2, 32, 48), (1, 4609, 1, 1, 64, 16),
                                   (1, 4100, 1, 1, 128, 32)],
                         ids=lambda s: "x".join(map(str, s)))
def test_long_sequences_in_segments(shape, dtype, decay):
    """Few heads and many chunks: the walk is split and joined again. Decays
    that keep a state over segments, that end it within one, and that leave
    nothing of it after a chunk."""
    *x, h0 = make(*shape, dtype, seed=17)
    x[3].mul_({"slow": 0.02, "fast": 1.0, "gone": 100.0}[decay])
    o, hT = forward(x, h0)
    ro, rS = delta_ref(*x, 0.125, h0)
    check(o, ro, "o")
    check(hT, rS, "hT")
    if decay == "slow" or shape[1] == 4200:
        g = torch.Generator().manual_seed(2)
        do = torch.randn(x[2].shape, generator=g).to(dtype).cuda()
        dhT = torch.randn(h0.shape, generator=g).cuda()
        got = backward(x, do, h0, dhT)
        ref = delta_ref(*x, 0.125, h0, do=do, dhT=dhT)
        for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), got, ref):
            check(a, b, name)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_packed_long_and_short(dtype):
    """Packed sequences of which one is split into segments."""
    cu = [0, 1, 4300, 4300, 4400, 8700]
    *x, h0 = make(1, cu[-1], 1, 1, 32, 32, dtype, seed=18, n=5)
    x[3].mul_(0.05)
    o, hT = forward(x, h0, cu)
    ro, rS = delta_ref(*x, 0.125, h0, cu)
    check(o, ro, "o")
    check(hT, rS, "hT")
    do = torch.randn(x[2].shape, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    got = backward(x, do, h0, h0, cu)
    ref = delta_ref(*x, 0.125, h0, cu, do=do, dhT=h0)
    for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), got, ref):
        check(a, b, name)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(48, 130, 1, 3, 128, 128), (48, 65, 3, 3, 104, 120),
                                   (2, 9000, 1, 4, 128, 128)],
                         ids=lambda s: "x".join(map(str, s)))
def test_many_wide_states(shape, dtype):
    """So many states of 128 rows that the waves of a workgroup share their
    operands, whole sequences and segments, with partial chunks and columns."""
    *x, h0 = make(*shape, dtype, seed=31)
    if shape[1] > 1000:
        x[3].mul_(0.05)
    o, hT = forward(x, h0)
    g = torch.Generator().manual_seed(3)
    do = torch.randn(x[2].shape, generator=g).to(dtype).cuda()
    dhT = torch.randn(h0.shape, generator=g).cuda()
    got = backward(x, do, h0, dhT)
    ro, rS = delta_ref(*x, 0.125, h0)
    check(o, ro, "o")
    check(hT, rS, "hT")
    ref = delta_ref(*x, 0.125, h0, do=do, dhT=dhT)
    for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), got, ref):
        check(a, b, name)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(96, 130, 1, 3, 64, 64), (96, 65, 3, 3, 32, 56),
                                   (96, 70, 1, 3, 112, 64), (2, 9000, 1, 8, 48, 64)],
                         ids=lambda s: "x".join(map(str, s)))
def test_many_states(shape, dtype):
    """As above with four tiles of columns, states of every padded height."""
    *x, h0 = make(*shape, dtype, seed=37)
    if shape[1] > 1000:
        x[3].mul_(0.05)
    o, hT = forward(x, h0)
    do = torch.randn(x[2].shape, generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    got = backward(x, do, h0, h0)
    ro, rS = delta_ref(*x, 0.125, h0)
    check(o, ro, "o")
    check(hT, rS, "hT")
    ref = delta_ref(*x, 0.125, h0, do=do, dhT=h0)
    for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), got, ref):
        check(a, b, name)


@pytest.mark.parametrize("size", [1e-12, 1e12])
def test_values_of_any_size(size):
    """Values and gradients far from 1, and one that is far from the rest."""
    *x, h0 = make(1, 300, 1, 1, 64, 32, F32, seed=19)
    x[2].mul_(size)
    x[2][0, 100, 0, 3] *= 1e4
    h0.mul_(size)
    do = size * torch.randn(x[2].shape, generator=torch.Generator().manual_seed(1)).cuda()
    o, hT = forward(x, h0)
    ro, rS = delta_ref(*x, 0.125, h0)
    check(o, ro, "o")
    check(hT, rS, "hT")
    got = backward(x, do, h0)
    ref = delta_ref(*x, 0.125, h0, do=do)
    for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), got, ref):
        check(a, b, name)


def test_keys_that_repeat():
    """All keys of a head equal and beta 1: the triangular matrix of a chunk
    is the worst conditioned one that unit keys give."""
    q, k, v, g, beta, h0 = make(1, 200, 1, 1, 64, 64, F32, seed=7, alike=1e6)
    beta.fill_(1.0)
    g.fill_(-0.01)
    o, hT = forward([q, k, v, g, beta], h0)
    ro, rS = delta_ref(q, k, v, g, beta, 0.125, h0)
    check(o, ro, "o")
    check(hT, rS, "hT")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_calls_continue_each_other(dtype):
    *x, h0 = make(2, 200, 1, 2, 64, 64, dtype, seed=8)
    ro, rS = delta_ref(*x, 0.125, h0)
    cut = 77
    a, mid = forward([t[:, :cut].contiguous() for t in x], h0)
    b, end = forward([t[:, cut:].contiguous() for t in x], mid)
    check(torch.cat([a, b], 1), ro, "o")
    check(end, rS, "hT")


def test_gradients_against_differences():
    """Central differences of the library's own forward in float32."""
    *x, h0 = make(1, 70, 1, 2, 16, 16, F32, seed=9)
    g = torch.Generator().manual_seed(3)
    do, dhT = torch.randn(x[2].shape, generator=g).cuda(), torch.randn(h0.shape, generator=g).cuda()
    got = backward(x, do, h0, dhT)
    def loss(y, s):
        o, hT = forward(y, s)
        return float((o.double() * do).sum() + (hT.double() * dhT).sum())
    # the step h costs h^2 / 6 of a third derivative (here below 30 in size)
    # and the forward's rounding, 1e-6 of |o| |do| ~ 30 at most, over 2 h
    h = 1e-2
    for i in range(6):
        d = torch.randn((x + [h0])[i].shape, generator=g).cuda()
        d /= d.norm()
        vals = []
        for sign in (1, -1):
            y = [t.clone() for t in x + [h0]]
            y[i] += sign * h * d
            vals.append(loss(y[:5], y[5]))
        want = (vals[0] - vals[1]) / (2 * h)
        have = float((got[i].double() * d).sum())
        assert abs(want - have) <= 1e-2 * max(1.0, abs(want)), (i, want, have)


def test_packed_values_outside_the_rule_stay_inside():
    """Decreasing or too large cu_seqlens: no access leaves the tensors (their
    surroundings keep their values)."""
    *x, _ = make(1, 100, 1, 1, 32, 32, F32)
    for cu in ([0, 80, 30, 100], [50, 500, 20, 7], [-5, 40, 1 << 30, 99]):
        room = torch.full((3, 100 * 32), 7.0, device="cuda")
        o = room[1].view(1, 100, 1, 32)
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        vmb.vmb_gated_delta_fwd(*x, o, cu_seqlens=c)
        torch.cuda.synchronize()
        assert (room[0] == 7).all() and (room[2] == 7).all()


def test_not_finite_stays_in_its_sequence():
    cu = [0, 100, 170, 200]
    *x, h0 = make(1, 200, 1, 2, 32, 32, BF16, n=3)
    clean, _ = forward(x, h0, cu)
    x[2][:, 150, 0, 3] = float("nan")
    x[1][:, 169] = float("inf")
    o, hT = forward(x, h0, cu)
    assert torch.equal(o[:, :100], clean[:, :100]) and torch.equal(o[:, 170:], clean[:, 170:])
    assert torch.isnan(o[:, 150:170, 0, 3]).all() and torch.isnan(hT[1]).any()
    assert torch.isfinite(hT[0]).all() and torch.isfinite(hT[2]).all()


def step(x, state, slots=None, scale=0.125):
    o = torch.full(x[2].shape, float("nan"), dtype=x[2].dtype, device="cuda")
    s = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
    vmb.vmb_gated_delta_step(*x, state, o, slots=s, scale=scale)
    torch.cuda.synchronize()
    return o


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 8, 8), (3, 1, 2, 4, 64, 64), (2, 5, 1, 3, 48, 80),
                                   (1, 2, 1, 1, 128, 128), (5, 3, 1, 2, 32, 256),
                                   (2, 1, 1, 1, 120, 136)],
                         ids=lambda s: "x".join(map(str, s)))
def test_step(shape, dtype):
    *x, h0 = make(*shape, dtype, seed=11)
    ro, rS = delta_ref(*x, 0.125, h0)
    state = h0.clone()
    o = step(x, state)
    check(o, ro, f"o {shape}")
    check(state, rS, f"state {shape}")


def test_step_slots():
    """Rows name their states; rows without one are skipped and write zeros."""
    *x, pool = make(5, 2, 1, 2, 64, 64, BF16, seed=12, n=9)
    slots = [7, -1, 0, 9, 3]
    state = pool.clone()
    o = step(x, state, slots)
    live = [0, 2, 4]
    sel = [t[live].contiguous() for t in x]
    ro, rS = delta_ref(*sel, 0.125, pool[[7, 0, 3]])
    check(o[live], ro, "o")
    check(state[[7, 0, 3]], rS, "state")
    assert not o[[1, 3]].any()
    rest = [1, 2, 4, 5, 6, 8]
    assert torch.equal(state[rest], pool[rest])


def test_step_views_and_zero_decay():
    B, hk, hv, d = 3, 1, 2, 32
    *x, pool = make(B, 1, hk, hv, d, d, F32, seed=13)
    x[3][0] = -float("inf")
    wide = torch.cat([t.flatten(2) for t in x[:3]], -1)
    q, k = wide[..., :d].unflatten(-1, (1, d)), wide[..., d:2 * d].unflatten(-1, (1, d))
    v = wide[..., 2 * d:].unflatten(-1, (hv, d))
    state = pool.clone()
    o = step([q, k, v] + x[3:], state)
    ro, rS = delta_ref(*x, 0.125, pool)
    check(o, ro, "o")
    check(state, rS, "state")


def test_steps_follow_a_chunked_call():
    """Serving: a map's tokens chunked, then single tokens."""
    *x, _ = make(2, 90, 1, 2, 64, 64, BF16, seed=14)
    ro, rS = delta_ref(*x, 0.125)
    o, state = forward([t[:, :80].contiguous() for t in x])
    outs = [o]
    for t in range(80, 90):
        outs.append(step([y[:, t:t + 1].contiguous() for y in x], state))
    check(torch.cat(outs, 1), ro, "o")
    check(state, rS, "state")


def test_side_stream_and_given_workspace():
    *x, h0 = make(1, 300, 1, 2, 64, 64, BF16, seed=15)
    want, _ = forward(x, h0)
    need = vmb.vmb_gated_delta_workspace_bytes(False, 1, 300, 1, 1, 2, 64, 64, BF16)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o = torch.empty_like(want)
    hT = torch.empty_like(h0)
    with torch.cuda.stream(side):
        vmb.vmb_gated_delta_fwd(*x, o, scale=0.125, h0=h0, hT=hT, workspace=ws)
    side.synchronize()
    assert torch.equal(o, want)


def test_captured_in_a_graph():
    """Forward, backward and step recorded once and replayed on new inputs."""
    *x, h0 = make(1, 200, 1, 2, 64, 64, BF16, seed=16)
    do = torch.randn(x[2].shape, device="cuda").to(BF16)
    o, hT = torch.empty_like(x[2]), torch.empty_like(h0)
    out = [torch.empty_like(t) for t in x]
    state, so = h0.clone(), torch.empty_like(x[2][:, :1])
    size = (1, 200, 1, 1, 2, 64, 64, BF16)
    ws = [torch.empty(vmb.vmb_gated_delta_workspace_bytes(b, *size), dtype=torch.uint8,
                      device="cuda") for b in (False, True)]
    first = [t[:, :1].contiguous() for t in x]

    def run():
        vmb.vmb_gated_delta_fwd(*x, o, h0=h0, hT=hT, workspace=ws[0])
        vmb.vmb_gated_delta_bwd(*x, do, *out, h0=h0, workspace=ws[1])
        vmb.vmb_gated_delta_step(*first, state, so)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(3):
        x[2].copy_(torch.randn(x[2].shape, device="cuda"))
        before = state.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (o, hT, *out, state)]
        state.copy_(before)
        run()
        torch.cuda.synchronize()
        for a, b in zip(got, (o, hT, *out, state)):
            assert torch.equal(a, b), i
