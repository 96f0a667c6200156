"""Shared links: the range of the values, and outputs where the parts of a row lie far apart."""
import numpy as np
import pytest
import torch

import link_model as L
from paper_2602_01519_amd import pic

pytestmark = pytest.mark.gpu


def group_over(k, v, n, q_len, q, hq, scale, **kw):
    """out, lse of n requests of q_len tokens that share one chunk and have no keys of their own."""
    hkv, d = k.shape[1:]
    with pic.Store(pic.GQA, pic.BF16, hkv, d, d, (len(k) + 63) // 64 * 64) as store:
        store.put(1, len(k), k, v, L.stream())
        out, lse = torch.full_like(q, 7.0), torch.zeros(len(q), hq, dtype=torch.float32, device="cuda")
        pic.link_shared(store, [0, n], [0, 1], [1], [0] * (n + 1), [], L.offsets([q_len] * n), None, hq, q, None, None,
                        scale, out, lse, stream=L.stream(), **kw)
        torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("q_len,n", [(5, 3), (8, 4), (20, 1)])
@pytest.mark.parametrize("sign", [1, -1])
def test_halves_of_a_block_that_pass_the_range_only_together(q_len, n, sign):
    """64-wide heads, groups of 60..128 rows, whose two halves of each tile's keys are summed apart. Over a
    first tile of logits 0 the next one's are 41 (2^59.15): a half is 32 x 2^59.15 x 1.375 x 2^63 =
    2^127.61, within fp32's range, both are not; the output is 1.375 x 2^63 but for the first tile's share, 2^-59 of
    that. A probability is off by half a bf16 step, 2^-8 of it, exponents and fp32 sums by less than 2^-11, the output by
    half a step."""
    k = torch.zeros(128, 2, 64, dtype=torch.bfloat16, device="cuda")
    k[64:, :, 0] = 41.0
    v = torch.ones_like(k)
    v[64:] = sign * 1.375 * 2.0 ** 63
    v[64:, :, 1::2] *= -1
    q = torch.zeros(n * q_len, 8, 64, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 8.0
    out, lse = group_over(k, v, n, q_len, q, 8, 0.125)
    ref, ref_lse = L.attend(q, k, v, 0.125)
    over = float(((out.double() - ref).abs() - ref.abs() * (2.0 ** -7 + 2.0 ** -11)).max())
    assert over <= 0
    off = float((lse.double() - ref_lse).abs().max())
    assert off <= 2.0 ** -11


@pytest.mark.parametrize("q_len,n,docs", [(1, 3, 700), (1, 70, 700), (3, 4, 130), (6, 3, 700), (40, 3, 700), (1, 160, 25001)])
def test_wide_heads_up_to_the_stated_range(q_len, n, docs):
    """128-wide heads: values up to 2^61 / T, T the 64-token tiles that a row sees, over a first tile of logits 0
    and others 40 above it (2^57.7, which no maximum follows: a lane's 32 probabilities stay below 2^64). A
    probability is off by half a bf16 step, 2^-8 of it, exponents and fp32 sums of up to 25,200 keys of one
    size by less than 2^-9, the output by half a step."""
    rng = np.random.default_rng(q_len + n)
    own = q_len + 30
    most = 2.0 ** (61 - int(np.ceil(np.log2((docs + 63) // 64 + (own + 63) // 64))))
    big = lambda *s: (L.draw(rng, pic.F32, *s).clamp(-2, 2) * (most / 2)).bfloat16()  # noqa: E731
    k = torch.zeros(docs, 2, 128, dtype=torch.bfloat16, device="cuda")
    k[64:, :, 0] = 40.0
    v = big(docs, 2, 128)
    v[64:, :, :64] = v[64:, :, :64].abs()          # (sums of one sign in half of the columns)
    q = torch.zeros(n * q_len, 8, 128, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 8.0
    ko = torch.zeros(n * own, 2, 128, dtype=torch.bfloat16, device="cuda")
    ko[::3, :, 0] = 38.0
    vo = big(n * own, 2, 128)
    out, lse = torch.full_like(q, 7.0), torch.zeros(n * q_len, 8, dtype=torch.float32, device="cuda")
    with pic.Store(pic.GQA, pic.BF16, 2, 128, 128, (docs + 63) // 64 * 64) as store:
        store.put(1, docs, k, v, L.stream())
        pic.link_shared(store, [0, n], [0, 1], [1], [0] * (n + 1), [], L.offsets([q_len] * n), L.offsets([own] * n), 8, q,
                        ko, vo, 0.125, out, lse, stream=L.stream())
        torch.cuda.synchronize()
    finite = bool(torch.isfinite(out).all())
    assert finite
    over = off = -1.0
    for r in range(n):
        at, rows = slice(r * q_len, (r + 1) * q_len), slice(r * own, (r + 1) * own)
        kk, vv, seen = torch.cat([k, ko[rows]]), torch.cat([v, vo[rows]]), L.causal(q_len, own, docs)
        ref, z = L.attend(q[at], kk, vv, 0.125, seen)
        size, _ = L.attend(q[at], kk, vv.abs(), 0.125, seen)
        over = max(over, float(((out[at].double() - ref).abs() - size * (2.0 ** -8 + 2.0 ** -9) - ref.abs() * 2.0 ** -8).max() / most))
        off = max(off, float((lse[at].double() - z).abs().max()))
    assert over <= 0
    assert off <= 2.0 ** -9
