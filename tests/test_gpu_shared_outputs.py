"""Shared links: outputs and log-sum-exp where the logits of a row's parts (the group's rows, its request's own links and
own KV) lie far apart, and of large values over 128-wide heads.

Bounds. Queries and keys hold whole numbers, so that the logits before the scale are exact in fp32
sums. With P the error of a probability as the value product takes it (bf16: half a step, 2^-8 of it), an
output is off by P sum p |v|, by half a step of its type, and by what follows from fp32
arithmetic: the logits' scale and the maxima are rounded to 2^-24 of them, which moves a
probability 2^-D by D 2^-24 of itself at each join (of at most 16), less than 2^-20 in all
as D 2^-D < 1, and the sums of up to 330 keys by 330 x 2^-24: together less than 2^-14 of sum p |v|,
numerator and denominator counted. Probabilities below 2^-126 of the largest may be 0: 330 x 2 of them, over values up
to 64, are less than 2^-110 (where every other value is 0, that is all there is). MLA sums the probabilities as they are rounded: P twice, and 1.01 x 2^-8 in
the log-sum-exp.

The vector-ALU kernel (widths without a kernel of their own: "generic" below) multiplies the queries by the scale
first: each is rounded, and so is each of the d products' partial sums, up to S = scale sum |q_i k_i| in size. A
logit is off by at most (d + 2) 2^-24 S, a probability by as much of itself, an output by twice that of
sum p |v|, the log-sum-exp by it once."""
import numpy as np
import pytest
import torch

import link_model as L
from paper_2602_01519_amd import pic

pytestmark = pytest.mark.gpu

SCALE = 0.125
FAR = {"bf16-128": (pic.GQA, pic.BF16, 2, 128, 128, 4), "bf16-128-mha": (pic.GQA, pic.BF16, 3, 128, 128, 1),
       "bf16-64": (pic.GQA, pic.BF16, 2, 64, 64, 4), "f32-64": (pic.GQA, pic.F32, 2, 64, 64, 4),
       "f32-128": (pic.GQA, pic.F32, 1, 128, 128, 3), "f32-40": (pic.GQA, pic.F32, 2, 40, 24, 2),
       "bf16-96": (pic.GQA, pic.BF16, 2, 96, 96, 2), "mla": (pic.MLA, pic.BF16, 1, 576, 512, 16)}
GENERIC = ("f32-40", "bf16-96")


def far_batch(rng, kind, dtype, hkv, dk, dv, group, q_len, n=6):
    """Element 0 of queries and keys sets the parts apart: logits of up to 400, and of a few, in
    every order of the parts. out, lse, their references, sum p |v|, the group's share of the
    probabilities, and the largest scale sum |q_i k_i|."""
    hq, mla, t = hkv * group, kind == pic.MLA, L.TORCH[dtype]
    whole = lambda *s: torch.from_numpy(rng.integers(-2, 3, s)).to(t).cuda()  # noqa: E731

    def keys(m, first):
        k = whole(m, hkv, dk)
        k[:, :, 0] = torch.from_numpy(np.broadcast_to(first, m).copy()).to(t).cuda()[:, None]
        return k, (k[..., :dv] if mla else L.draw(rng, dtype, m, hkv, dv))

    shared = [keys(m, rng.integers(-3, 4, m)) for m in (130, 70)]
    mine = [keys(30, 0) for _ in range(n)]
    own_len = q_len + 3
    own = [keys(own_len, np.where(np.arange(own_len) % 2, 50, -50) if r % 2 else rng.integers(-2, 3, own_len)) for r in range(n)]
    q = whole(n * q_len, hq, dk)
    q[:, :, 0] = torch.from_numpy(rng.choice([0, 1, -1, 5, 64, -64], (n * q_len, hq))).to(t).cuda()
    out, lse = torch.full((len(q), hq, dv), 7.0, dtype=t, device="cuda"), torch.zeros(len(q), hq, dtype=torch.float32, device="cuda")
    with pic.Store(kind, dtype, hkv, dk, dv, 64 * 20) as store:
        for i, (k, v) in enumerate(shared + mine):
            store.put(i, len(k), k, None if mla else v, L.stream())
        ko = torch.cat([k for k, _ in own])
        vo = None if mla else torch.cat([v for _, v in own])
        pic.link_shared(store, [0, n], [0, 2], [0, 1], range(n + 1), range(2, 2 + n), L.offsets([q_len] * n),
                        L.offsets([own_len] * n), hq, q, ko, vo, SCALE, out, lse, stream=L.stream())
        torch.cuda.synchronize()
    refs, sizes, lses, weight, most = [], [], [], [], 0.0
    for r in range(n):
        ks, vs = (torch.cat([x[i] for x in shared + [mine[r], own[r]]]) for i in range(2))
        seen = L.causal(q_len, own_len, 230)
        at = q[r * q_len:(r + 1) * q_len]
        ref, z = L.attend(at, ks, vs, SCALE, seen)
        refs.append(ref)
        lses.append(z)
        sizes.append(L.attend(at, ks, vs.abs(), SCALE, seen)[0])
        weight.append(torch.exp(L.attend(at, ks[:200], vs[:200], SCALE)[1] - z))    # of the group's rows
        for h in range(hq):
            most = max(most, SCALE * float((at[:, h].double().abs() @ ks[:, h // group].double().abs().T.contiguous()).max()))
    return out, lse, torch.cat(refs), torch.cat(lses), torch.cat(sizes), torch.cat(weight), most


@pytest.mark.parametrize("name,q_len", [("bf16-128", 1), ("bf16-128", 6), ("bf16-128", 40), ("bf16-128-mha", 1), ("bf16-64", 1),
                                        ("bf16-64", 9), ("bf16-64", 40), ("f32-64", 1), ("f32-64", 6), ("f32-128", 1),
                                        ("f32-40", 2), ("bf16-96", 1), ("mla", 1), ("mla", 5)])
def test_parts_far_apart(name, q_len):
    shape = FAR[name]
    rng = np.random.default_rng(6 + q_len)
    out, lse, ref, z, size, weight, most = far_batch(rng, *shape, q_len)
    # (either part alone, and both)
    alone, none, both = (bool(x.any()) for x in (weight > 0.99, weight < 1e-6, (weight > 0.2) & (weight < 0.9)))
    assert alone and none and both
    p, step = (2.0 ** -8, 2.0 ** -8) if shape[1] == pic.BF16 else (0.0, 2.0 ** -24)
    mla = shape[0] == pic.MLA
    logit = (shape[3] + 2) * 2.0 ** -24 * most if name in GENERIC else 0.0
    finite = bool(torch.isfinite(out).all())
    assert finite
    over = float(((out.double() - ref).abs() - (size * ((2.02 if mla else 1.0) * p + 2.0 ** -14 + 2 * logit) + ref.abs() * step + 2.0 ** -110)).max())
    assert over <= 0
    bound = (1.01 * p if mla else 0.0) + 2.0 ** -14 + logit + 2.0 ** -22 * z.abs()
    over = float(((lse.double() - z).abs() - bound).max())
    assert over <= 0
