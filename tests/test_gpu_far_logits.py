"""Logits far from zero, in the kernels of the bf16 stores: a row's probabilities must not be
formed against a maximum of zero, where those of logits below -103 are all 0 in fp32.

Tolerances. The kernels of the bf16 128-wide GQA and MLA stores sum the probabilities as they
are rounded to bf16, p (1 + d), |d| <= 2^-8, in the products and in the sum they are divided by:
each of the two moves an output by at most 2^-8 W (W as in fp4_model.py, whose other terms are
the same), together and with the products of such errors less than 2.05 times its tolerance.
The logarithm of the sum moves by less than 1.01 * 2^-8."""
import numpy as np
import pytest
import torch

import fp4_model as M
from paper_2602_01519_amd import pic

pytestmark = pytest.mark.gpu

GQA, MLA = dict(kind=pic.GQA, hkv=2, dk=128, dv=128), dict(kind=pic.MLA, hkv=1, dk=576, dv=512)


def dev(x):
    return torch.from_numpy(M.bits(x)).cuda()


def host(t):
    return (t.cpu().numpy().view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def run(shape, hq, chunks, links, q_len, q, own_len, own, scale, limits=None, decode=False, splits=0):
    """out, lse of one call; chunks [(k, v)], links: chunk numbers per request."""
    st = torch.cuda.current_stream().cuda_stream
    off = lambda x: np.concatenate([[0], np.cumsum(x)]).astype(np.int32)  # noqa: E731
    mla = shape["kind"] == pic.MLA
    cap = sum((len(k) + 63) // 64 * 64 for k, _ in chunks)
    with pic.Store(shape["kind"], pic.BF16, shape["hkv"], shape["dk"], shape["dv"], cap) as store:
        for i, (k, v) in enumerate(chunks):
            store.put(i, len(k), dev(k), None if mla else dev(v), st)
        out = torch.full((len(q), hq, shape["dv"]), 77, dtype=torch.int16, device="cuda")
        lse = torch.full((len(q), hq), 5.0, dtype=torch.float32, device="cuda")
        ks = None if own is None else dev(own[0])
        vs = None if own is None or mla else dev(own[1])
        kw = dict(num_splits=splits) if decode else {}
        (pic.link_decode if decode else pic.link_attn)(
            store, off([len(l) for l in links]), [c for l in links for c in l], off(q_len),
            None if own is None else off(own_len), hq, dev(q), ks, vs, scale, out, lse, stream=st,
            q_doc_limits=limits, **kw)
        torch.cuda.synchronize()
        return host(out), lse.cpu().numpy().astype(np.float64)


def check(shape, hq, chunks, links, q_len, q, own_len, own, scale, limits, got):
    kept = dict(enumerate(chunks))
    off = lambda x: np.concatenate([[0], np.cumsum(x)])  # noqa: E731
    ko, vo = (None, None) if own is None else own
    ro, rl, to, tl = [], [], [], []
    q0, s0 = off(q_len), off(own_len) if own is not None else None
    for r, l in enumerate(links):
        k = [kept[c][0] for c in l]
        v = [kept[c][1] for c in l]
        doc, ls = sum(len(x) for x in k), 0
        if own is not None:
            ls = own_len[r]
            k.append(ko[s0[r]:s0[r] + ls])
            v.append(vo[s0[r]:s0[r] + ls])
        seen = np.zeros((q_len[r], doc + ls), bool)
        for i in range(q_len[r]):
            seen[i, :doc if limits is None else limits[q0[r] + i]] = True
            seen[i, doc:doc + i + 1 + ls - q_len[r]] = True
        # fp4_model.attend pairs widths of q and v: columns of zeros make them alike
        kk, vv = np.concatenate(k), np.concatenate(v)
        qq = q[q0[r]:q0[r + 1]]
        a = M.attend(qq, kk, np.pad(vv, ((0, 0), (0, 0), (0, shape["dk"] - shape["dv"]))), scale, seen)
        for x, y in zip((ro, rl, to, tl), a):
            x.append(y[..., :shape["dv"]] if y.ndim == 3 else y)
    ro, rl, to, tl = (np.concatenate(x) for x in (ro, rl, to, tl))
    out, lse = got
    assert np.array_equal(np.isfinite(lse), np.isfinite(rl))
    f = np.isfinite(rl)
    assert (np.abs(lse[f] - rl[f]) <= tl[f] + 1.01 * 2.0 ** -8 + 2.0 ** -22 * np.abs(rl[f])).all(), \
        np.abs(lse[f] - rl[f]).max()
    over = np.abs(out - ro) - 2.05 * to
    assert not np.isnan(out).any() and (over <= 0).all(), f"out off its bound by {over.max()}"


# shape, query heads, chunk lengths, links, query tokens, own beyond the query (None: no own
# KV), limits, decode, pieces
CASES = {
    "gqa_short": (GQA, 8, (70, 64, 130), [(0, 1), (2,), (1, 0, 2)], (3, 40, 1), (5, 0, 64), False, False, 0),
    "gqa_blocks": (GQA, 8, (70, 64, 130), [(0, 1), (2, 2)], (90, 70), (0, 33), False, False, 0),
    "gqa_cross": (GQA, 4, (200, 65), [(0, 1), (1,)], (150, 20), None, False, False, 0),
    "gqa_limits": (GQA, 8, (70, 64, 130), [(0, 1, 2), (2,)], (80, 20), None, True, False, 0),
    "gqa_limits_own": (GQA, 8, (70, 64, 130), [(0, 1, 2), (2,)], (20, 70), (0, 3), True, False, 0),
    "gqa_wide_decode": (GQA, 64, (300, 65), [(0, 1), (1, 0)], (2, 3), (0, 9), False, True, 3),
    "gqa_decode": (GQA, 8, (300, 65), [(0, 1), (1, 0)], (1, 2), (0, 9), False, True, 0),
    "mla_prefill": (MLA, 16, (70, 64, 130), [(0, 1), (2,), (1, 0, 2)], (3, 20, 1), (5, 0, 64), False, False, 0),
    "mla_cross": (MLA, 16, (200, 65), [(0, 1), (1,)], (9, 20), None, False, False, 0),
    "mla_limits": (MLA, 8, (70, 64, 130), [(0, 1, 2), (2,)], (20, 30), None, True, False, 0),
    "mla_decode": (MLA, 16, (300, 65), [(0, 1), (1, 0)], (1, 2), (0, 9), False, True, 3),
}


def inputs(name, seed):
    shape, hq, lens, links, q_len, extra, limited, decode, splits = CASES[name]
    rng = np.random.default_rng(seed + sum(map(ord, name)))
    dk, dv, hkv = shape["dk"], shape["dv"], shape["hkv"]

    def kv(n):
        k = M.bf16(rng.standard_normal((n, hkv, dk)))
        return k, k[..., :dv] if shape["kind"] == pic.MLA else M.bf16(rng.standard_normal((n, hkv, dv)))

    chunks = [kv(n) for n in lens]
    own_len = None if extra is None else [a + b for a, b in zip(q_len, extra)]
    own = None if extra is None else kv(sum(own_len))
    q = M.bf16(rng.standard_normal((sum(q_len), hq, dk)))
    limits = None
    if limited:
        limits = np.concatenate([rng.integers(0, sum(lens[c] for c in l) + 1, n) for l, n in zip(links, q_len)])
        limits[0] = 0
    return shape, hq, chunks, links, list(q_len), q, own_len, own, limits, decode, splits


@pytest.mark.parametrize("name", sorted(CASES))
@pytest.mark.parametrize("sign", [-1, 1])
def test_all_logits_far_from_zero(name, sign):
    """Every logit lies hundreds below (above) zero: one element of q and of each key gives a
    logit of 400, the others vary it."""
    shape, hq, chunks, links, q_len, q, own_len, own, limits, decode, splits = inputs(name, 1)
    scale = float(np.float32(shape["dk"] ** -0.5))

    def far(kv):
        k = kv[0].copy()
        k[..., shape["dk"] - 1] = M.bf16(sign * 400 / scale / 64)
        return k, k[..., :shape["dv"]] if shape["kind"] == pic.MLA else kv[1]

    q[..., shape["dk"] - 1] = 64
    chunks = [far(c) for c in chunks]
    own = None if own is None else far(own)
    print(name, flush=True)
    got = run(shape, hq, chunks, links, q_len, q, own_len, own, scale, limits, decode, splits)
    check(shape, hq, chunks, links, q_len, q, own_len, own, scale, limits, got)


@pytest.mark.parametrize("name", sorted(CASES))
@pytest.mark.parametrize("seed", [2, 3])
def test_logits_around_the_underflow(name, seed):
    """Whole logits from -107 to -99, each exact, in every order: what lies below -103 counts
    beside what lies above."""
    shape, hq, chunks, links, q_len, q, own_len, own, limits, decode, splits = inputs(name, seed)
    rng = np.random.default_rng(seed)

    def far(kv):
        k = kv[0].copy()
        k[..., shape["dk"] - 1] = -rng.integers(99, 108, k.shape[:2])
        # a first tile that underflows as a whole
        k[:64, :, shape["dk"] - 1] = -rng.integers(104, 108, k[:64].shape[:2])
        return k, k[..., :shape["dv"]] if shape["kind"] == pic.MLA else kv[1]

    q[...] = 0
    q[..., shape["dk"] - 1] = 1
    chunks = [far(c) for c in chunks]
    own = None if own is None else far(own)
    print(name, flush=True)
    got = run(shape, hq, chunks, links, q_len, q, own_len, own, 1.0, limits, decode, splits)
    check(shape, hq, chunks, links, q_len, q, own_len, own, 1.0, limits, got)
