"""Rotary positions: several tensors of one call, in place and not, and very many tokens."""
import math

import numpy as np
import pytest
import torch

from paper_2602_01519_amd import pic
from test_gpu_rope import check, frequencies, stream, to_dev, turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [2 ** 27 + 5])
def test_rotary_positions_of_many_tokens(n):
    """One pair per token, 2^24 workgroups of eight tokens and one more. Tolerance as in
    test_gpu_rope.py, the reference in 64 bits on the GPU, in slices."""
    x = torch.empty(n, 1, 2, dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    y = torch.full_like(x, 7.0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x.copy_(torch.randn(1 << 20, 1, 2, generator=gen, device="cuda").bfloat16().repeat(n // (1 << 20) + 1, 1, 1)[:n])
    with pic.Rope(pic.BF16, pic.ROPE_HALF, 2, 0, 2) as rope:
        rope.apply(n, pos, [(x, y, 1, 0, 0)], stream=stream())
    torch.cuda.synchronize()
    for a in range(0, n, 1 << 24):
        p, u = pos[a:a + (1 << 24)].double(), x[a:a + (1 << 24), 0].double()
        turns = p / (2 * math.pi)
        angle = 2 * math.pi * (turns - torch.round(turns))
        c, s = torch.cos(angle), torch.sin(angle)
        ref = torch.stack([c * u[:, 0] - s * u[:, 1], s * u[:, 0] + c * u[:, 1]], 1)
        tol = (2.0 ** -22 + 2.0 ** -23) * u.abs().sum(1, keepdim=True) + 2.0 ** -8 * ref.abs()
        assert bool(((y[a:a + (1 << 24), 0].double() - ref).abs() <= tol).all()), f"tokens from {a}"
