"""A token mixer for channels-last maps from the library's operators: group norm
with SiLU, one product to queries, keys and values, rotary positions on rows and
columns with unit-length heads, the gated delta rule over the tokens, a product
back and the residual.

    python examples/delta_mixer.py

trains one block on a map-to-map task for a few steps (forward and backward of
all three operators) and then streams frames through it, the state carried from
frame to frame: whole frames by the chunked form, the last one token by token.
PyTorch supplies memory, the products, the optimizer and the chain rule between
the calls; data and weights are random.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2412_16602_amd import vmb  # noqa: E402


class GroupNormSilu(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, groups, eps):
        y = torch.empty_like(x)
        mean = torch.empty(x.shape[0], groups, device=x.device)
        rstd = torch.empty_like(mean)
        vmb.vmb_group_norm_act_fwd(x, gamma, beta, groups, eps, vmb.VMB_ACT_SILU, y, mean, rstd)
        ctx.save_for_backward(x, gamma, beta, mean, rstd)
        ctx.groups = groups
        return y

    @staticmethod
    def backward(ctx, dy):
        x, gamma, beta, mean, rstd = ctx.saved_tensors
        dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
        vmb.vmb_group_norm_act_bwd(dy.contiguous(), x, gamma, beta, mean, rstd, ctx.groups,
                                   vmb.VMB_ACT_SILU, dx, dgamma, dbeta)
        return dx, dgamma, dbeta, None, None


class UnitRotary(torch.autograd.Function):
    """Queries and keys, scaled to unit length and turned by their positions."""

    @staticmethod
    def forward(ctx, q, k, positions, inv_freq, sections, eps):
        yq, yk = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
        vmb.vmb_axis_rotary_fwd(q, k, positions, inv_freq, sections, yq, yk, norm_eps=eps)
        ctx.save_for_backward(q, k, positions, inv_freq)
        ctx.sections, ctx.eps = sections, eps
        return yq, yk

    @staticmethod
    def backward(ctx, d_yq, d_yk):
        q, k, positions, inv_freq = ctx.saved_tensors
        d_yq, d_yk = d_yq.contiguous(), d_yk.contiguous()
        d_q, d_k = torch.empty_like(d_yq), torch.empty_like(d_yk)
        vmb.vmb_axis_rotary_bwd(d_yq, d_yk, q, k, positions, inv_freq, ctx.sections, d_q, d_k,
                                norm_eps=ctx.eps)
        return d_q, d_k, None, None, None, None


class GatedDelta(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, g, beta):
        o = torch.empty(v.shape, dtype=v.dtype, device=v.device)
        vmb.vmb_gated_delta_fwd(q, k, v, g, beta, o)
        ctx.save_for_backward(q, k, v, g, beta)
        return o

    @staticmethod
    def backward(ctx, do):
        x = ctx.saved_tensors
        grads = [torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in x]
        vmb.vmb_gated_delta_bwd(*x, do.contiguous(), *grads)
        return tuple(grads)


class DeltaMixer(torch.nn.Module):
    """x [batch, H, W, channels] -> the same shape."""

    def __init__(self, channels=192, heads=3, head_dim=64, groups=32, dtype=torch.bfloat16):
        super().__init__()
        self.heads, self.head_dim, self.groups = heads, head_dim, groups
        width = heads * head_dim
        self.gamma = torch.nn.Parameter(torch.ones(channels))
        self.beta = torch.nn.Parameter(torch.zeros(channels))
        self.qkv = torch.nn.Linear(channels, 3 * width, bias=False, dtype=dtype)
        self.gates = torch.nn.Linear(channels, 2 * heads, dtype=dtype)
        self.out = torch.nn.Linear(width, channels, bias=False, dtype=dtype)
        pairs = head_dim // 4  # for each of row and column; they fill the head
        self.sections = (pairs, pairs)
        turn = 100.0 ** (-torch.arange(pairs, dtype=torch.float32) / pairs)
        self.register_buffer("inv_freq", torch.cat([turn, turn]))

    def positions(self, H, W):
        rows, cols = torch.meshgrid(torch.arange(H), torch.arange(W), indexing="ij")
        p = torch.stack([rows, cols], -1).reshape(1, H * W, 2)
        return p.to(device=self.inv_freq.device, dtype=torch.int32).contiguous()

    def inputs(self, x):
        """What the recurrence takes: q, k of unit length, v (a view of the
        product), log decays and write strengths."""
        B, H, W, C = x.shape
        y = GroupNormSilu.apply(x, self.gamma, self.beta, self.groups, 1e-5).reshape(B, H * W, C)
        q, k, v = self.qkv(y).unflatten(-1, (3, self.heads, self.head_dim)).unbind(2)
        q, k = UnitRotary.apply(q, k, self.positions(H, W), self.inv_freq, self.sections, 1e-6)
        decay, write = self.gates(y).float().chunk(2, -1)
        g = -0.1 * torch.nn.functional.softplus(decay)
        return q, k, v, g.contiguous(), torch.sigmoid(write).contiguous()

    def mix(self, x, o):
        return x + self.out(o.flatten(2)).reshape(x.shape)

    def forward(self, x):
        return self.mix(x, GatedDelta.apply(*self.inputs(x)))

    def new_state(self, batch):
        return torch.zeros(batch, self.heads, self.head_dim, self.head_dim,
                           device=self.inv_freq.device)

    @torch.no_grad()
    def frame(self, x, state, single_tokens=False):
        """One frame of a stream; state [batch, heads, d, d] is updated."""
        q, k, v, g, beta = self.inputs(x)
        o = torch.empty(v.shape, dtype=v.dtype, device=v.device)
        if single_tokens:
            one = torch.empty(o[:, :1].shape, dtype=o.dtype, device=o.device)
            for t in range(v.shape[1]):
                tok = [a[:, t:t + 1].contiguous() for a in (q, k, v, g, beta)]
                vmb.vmb_gated_delta_step(*tok, state, one)
                o[:, t:t + 1] = one
        else:
            vmb.vmb_gated_delta_fwd(q, k, v, g, beta, o, h0=state.clone(), hT=state)
        return self.mix(x, o)


def train(steps=30, batch=4, side=14, dtype=torch.bfloat16, log=print):
    """Learns a fixed map of each token's channels, which only the path through
    the operators can add; returns the losses and the block."""
    torch.manual_seed(0)
    block = DeltaMixer(dtype=dtype).cuda()
    mixture = torch.randn(192, 192, device="cuda") / 14.0
    best = torch.optim.Adam(block.parameters(), lr=2e-3)
    losses = []
    for i in range(steps):
        x = torch.randn(batch, side, side, 192, device="cuda")
        target = x + torch.nn.functional.silu(x) @ mixture
        loss = torch.nn.functional.mse_loss(block(x.to(dtype)).float(), target)
        best.zero_grad()
        loss.backward()
        best.step()
        losses.append(float(loss.detach()))
        if i % 10 == 0 or i == steps - 1:
            log(f"step {i:3d}  loss {losses[-1]:.5f}")
    return losses, block


def stream(block, frames=3, batch=2, side=7, dtype=torch.bfloat16, log=print):
    """Frames in a row; the last one twice from the same state, whole and token
    by token. Returns the two outputs and the two states."""
    torch.manual_seed(1)
    state = block.new_state(batch)
    for _ in range(frames - 1):
        block.frame(torch.randn(batch, side, side, 192, device="cuda").to(dtype), state)
    x = torch.randn(batch, side, side, 192, device="cuda").to(dtype)
    again = state.clone()
    whole = block.frame(x, state)
    single = block.frame(x, again, single_tokens=True)
    log(f"{frames} frames of {side} x {side}: largest difference of the last one, whole and "
        f"token by token: {float((whole.float() - single.float()).abs().max()):.2e}")
    return whole, single, state, again


if __name__ == "__main__":
    _, trained = train()
    stream(trained)
