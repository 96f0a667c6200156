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


@pytest.mark.parametrize("dtype", [pic.F32, pic.BF16])
@pytest.mark.parametrize("layout", [pic.ROPE_HALF, pic.ROPE_INTERLEAVED])
@pytest.mark.parametrize("n", [1, 7, 1500])
def test_four_tensors_in_place_and_not(dtype, layout, n):
    """Four tensors of different head counts in one call: two in place, one of them a slice of
    wider rows, and two not, with elements that are not turned on both sides of those that are."""
    rng = np.random.default_rng(n)
    width, at, rot, heads = 90, 21, 46, (1, 12, 5, 3)
    pos = rng.integers(-1000, 200000, n).astype(np.int32)
    wide = to_dev(rng.standard_normal((n, 15, width)), dtype)
    x = [to_dev(rng.standard_normal((n, 1, width)), dtype), wide[:, 2:14], to_dev(rng.standard_normal((n, 5, width)), dtype),
         to_dev(rng.standard_normal((n, 3, width)), dtype)]
    before, wide_before = [t.clone() for t in x], wide.clone()
    out = [x[0], x[1], torch.full_like(x[2], 7.0), torch.full((n, 4, width), 7.0, dtype=x[3].dtype, device="cuda")]
    with pic.Rope(dtype, layout, width, at, rot) as rope:
        rope.apply(n, torch.from_numpy(pos).cuda(),
                   [(x[0], out[0], 1, 0, 0), (x[1], out[1], 12, 15 * width, 15 * width), (x[2], out[2], 5, 0, 0),
                    (x[3], out[3], 3, 0, 4 * width)], stream=stream())
        torch.cuda.synchronize()
    part = np.ones(width, bool)
    part[at:at + rot] = False
    for b, y, h in zip(before, out, heads):
        ref, size = turned(b.double().cpu().numpy(), pos, frequencies(rot, 10000.0), 1.0, layout == pic.ROPE_HALF, at,
                           rot, False)
        check(y[:, :h], ref, size, dtype)
        assert torch.equal(y[:, :h][..., part], b[..., part])
    assert torch.equal(x[2], before[2]) and torch.equal(x[3], before[3])
    assert bool((out[3][:, 3] == 7.0).all())
    assert torch.equal(wide[:, :2], wide_before[:, :2]) and torch.equal(wide[:, 14:], wide_before[:, 14:])
