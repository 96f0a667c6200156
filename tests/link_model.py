"""Link attention from its definition in 64 bits, and seeded stores and batches (plain torch; no
test_ prefix)."""
import numpy as np
import torch

import parity_gate as G
from paper_2602_01519_amd import pic

TORCH = {pic.F32: torch.float32, pic.BF16: torch.bfloat16}


def stream():
    return torch.cuda.current_stream().cuda_stream


def offsets(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def draw(rng, dtype, *shape):
    return torch.from_numpy(rng.standard_normal(shape)).to(TORCH[dtype]).cuda()


def attend(q, k, v, scale, seen=None):
    """q [tokens][heads][d_k], k [keys][kv heads][d_k], v [keys][kv heads][d_v], seen [tokens][keys]:
    output and log-sum-exp in 64 bits."""
    n, hq, _ = q.shape
    hkv = k.shape[1]
    out = torch.zeros(n, hq, v.shape[2], dtype=torch.float64, device=q.device)
    lse = torch.full((n, hq), -float("inf"), dtype=torch.float64, device=q.device)
    if not len(k) or not n:
        return out, lse
    for h in range(hq):
        kh, vh = k[:, h // (hq // hkv)].double(), v[:, h // (hq // hkv)].double()
        s = scale * (q[:, h].double() @ kh.T.contiguous())
        if seen is not None:
            s = torch.where(seen, s, -float("inf"))
        lse[:, h] = torch.logsumexp(s, -1)
        some = torch.isfinite(lse[:, h])
        w = torch.exp(s - torch.where(some, lse[:, h], torch.zeros_like(lse[:, h]))[:, None])
        out[:, h] = torch.where(some[:, None], w @ vh, torch.zeros_like(out[:, h]))
    return out, lse


def causal(lq, ls, docs, limits=None):
    """seen [lq][docs + ls]: linked rows up to each token's limit, own keys bottom-right causal."""
    seen = torch.ones(lq, docs + ls, dtype=torch.bool)
    for i in range(lq):
        if limits is not None:
            seen[i, int(limits[i]):docs] = False
        if ls:
            seen[i, docs + ls - lq + i + 1:] = False
    return seen.cuda()


def check(dtype, out, lse, ref, ref_lse, label=""):
    """The parity bar of tests/parity_gate.py."""
    host = lambda x: x.double().cpu().numpy()  # noqa: E731
    bad = G.failures(G.F32 if dtype == pic.F32 else G.BF16, host(out), host(ref),
                     None if lse is None else host(lse), None if lse is None else host(ref_lse))
    assert not bad, f"{label}: {bad}"
