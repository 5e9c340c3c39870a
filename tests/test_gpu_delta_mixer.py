"""examples/delta_mixer.py: the three operators in one block, trained for a few
steps and run as a stream."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))


def quiet(_):
    pass


def test_a_block_learns():
    import delta_mixer
    losses, _ = delta_mixer.train(steps=30, log=quiet)
    assert all(x == x for x in losses)
    assert sum(losses[-3:]) < 0.9 * sum(losses[:3])


def test_gradients_of_the_block_against_differences():
    """A directional difference of the whole block in fp32."""
    import delta_mixer
    torch.manual_seed(2)
    block = delta_mixer.DeltaMixer(channels=64, heads=2, head_dim=16, groups=8,
                                   dtype=torch.float32).cuda()
    x = torch.randn(2, 5, 7, 64, device="cuda")
    w = torch.randn_like(x)
    for name, p in [("x", x.requires_grad_(True))] + list(block.named_parameters()):
        block.zero_grad()
        x.grad = None
        (block(x) * w).sum().backward()
        d = torch.randn_like(p)
        d /= d.norm()
        slope = float((p.grad.double() * d.double()).sum())
        eps = 2e-2
        with torch.no_grad():
            p += eps * d
            up = float((block(x).double() * w.double()).sum())
            p -= 2 * eps * d
            down = float((block(x).double() * w.double()).sum())
            p += eps * d
        # the difference's own error: eps^2 of a third derivative, and the
        # rounding of outputs of size 1 in fp32, sqrt(4480) 2^-24 / eps
        scale = float(p.grad.double().norm())
        assert abs((up - down) / (2 * eps) - slope) <= 1e-2 * scale + 1e-3, name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_stream_whole_and_by_tokens(dtype):
    import delta_mixer
    torch.manual_seed(3)
    block = delta_mixer.DeltaMixer(dtype=dtype).cuda()
    whole, single, state, again = delta_mixer.stream(block, dtype=dtype, log=quiet)
    # each side rounds o once (bf16: half of 2^-8 of it) before the product back
    tol = 2e-5 if dtype == torch.float32 else 1e-2
    assert float((whole - single).float().norm()) <= tol * float(whole.float().norm())
    assert float((state - again).norm()) <= 2e-5 * float(state.norm())
