"""4-bit caches whose values are as large as the format holds (infinities are kept as
6 * 2^125): sums of them leave the fp32 range although the outputs, their means, do not.

Both sides are as in fp4_model.py, with a reference in 64 bits on the GPU. Its tolerances,
but for what a second pass over a piece of n keys loses: probabilities below 2^-126 of its unit,
which is at most 2 n times the largest one's, and outputs below 2^-126 in it. Both reach a
channel as its own values do: 2 n 2^-126 (n max|v| + 1), with n rounded up to whole tiles."""
import numpy as np
import pytest
import torch

import fp4_model as M
from paper_2602_01519_amd import pic
from test_gpu_fp4 import Call, ROWS_256

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def attend(q, k, v, scale, seen, tiles):
    """Rows q [m][d] of one kv head over k, v [n][d], seen [m][n], all in 64 bits on the GPU."""
    n, d = k.shape
    s = torch.where(seen, scale * (q @ k.T.contiguous()), -torch.inf)
    some = seen.any(1)
    top = torch.where(some, s.amax(1), 0.0)
    p = torch.exp(s - top[:, None])
    total = p.sum(1)
    w = p / torch.where(some, total, 1.0)[:, None]
    out = w @ v
    lse = torch.where(some, top + torch.log(torch.where(some, total, 1.0)), -torch.inf)
    size = torch.where(seen, scale * (q.abs() @ k.abs().T.contiguous()), 0.0).amax(1)
    logit = torch.where(seen, s.abs(), 0.0).amax(1)
    e = U * (d * size + 4 * logit + n + 48)
    unit = 2 * 64 * tiles * 2.0 ** -126
    tol = 2.0 ** -8 * out.abs() + (2.0 ** -8 + 4 * e[:, None]) * (w @ v.abs()) + \
        unit * (n * v.abs().amax(0) + 1)
    return out, lse, torch.where(some[:, None], tol, 0.0), torch.where(some, e + 4 * U * lse.abs(), 0.0)


def check(c, got):
    """A call's (out, lse) against the reference of every request and head."""
    out, lse = (torch.from_numpy(x).cuda() for x in got)
    gpu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    group = c.hq // c.hkv
    kept = {i: (gpu(M.stored(k)), gpu(M.stored(v))) for i, (k, v) in c.raw.items()}
    for r, ids in enumerate(c.links):
        q0, q1 = int(c.q_off[r]), int(c.q_off[r + 1])
        lq = q1 - q0
        if lq == 0:
            continue
        ks = [kept[i][0][a:] for i, a in zip(ids, c.starts[r])]
        vs = [kept[i][1][a:] for i, a in zip(ids, c.starts[r])]
        doc, ls = sum(len(x) for x in ks), 0
        tiles = sum((len(x) + 63) // 64 for x in ks)
        if c.own_off is not None:
            a, b = int(c.own_off[r]), int(c.own_off[r + 1])
            ls = b - a
            ks.append(gpu(c.k_own[a:b]))
            vs.append(gpu(c.v_own[a:b]))
            tiles += (ls + 63) // 64
        i = torch.arange(lq, device="cuda")[:, None]
        j = torch.arange(doc + ls, device="cuda")[None]
        far = torch.full((lq, 1), doc, device="cuda") if c.limits is None else \
            torch.from_numpy(np.asarray(c.limits[q0:q1], np.int64)).cuda()[:, None]
        seen = torch.where(j < doc, j < far, j - doc <= i + ls - lq).repeat_interleave(group, 0)
        if doc + ls == 0:
            assert bool((out[q0:q1] == 0).all()) and bool((lse[q0:q1] == -torch.inf).all())
            continue
        k, v = torch.cat(ks), torch.cat(vs)
        for h in range(c.hkv):
            heads = slice(h * group, (h + 1) * group)
            q = gpu(c.q[q0:q1, heads].reshape(lq * group, c.d))
            ro, rl, to, tl = attend(q, k[:, h].contiguous(), v[:, h].contiguous(), c.scale, seen, max(tiles, 1))
            o, l = out[q0:q1, heads].reshape(lq * group, c.d), lse[q0:q1, heads].reshape(-1)
            assert torch.equal(torch.isfinite(l), torch.isfinite(rl))
            f = torch.isfinite(rl)
            assert bool(((l - rl).abs()[f] <= tl[f]).all()), f"lse of request {r}, head {h}"
            over = (o - ro).abs() - to
            assert bool(torch.isfinite(o).all()) and bool((over <= 0).all()), \
                f"out of request {r}, head {h} off its bound by {float(over.max())}"


def large(c):
    """Large values in a few channels of the first block of every row; the others stay."""
    rng = np.random.default_rng(1)

    def spoil(v):
        v = v.copy()
        v[:, :, 5] = np.inf
        v[:, :, 6] = np.where(rng.random(v.shape[:2]) < 0.5, np.inf, -np.inf)
        v[::3, :, 7] = -1e38
        v[len(v) // 2, :, 20] = 3e38
        return M.bf16(v)

    c.raw = {i: (k, spoil(v)) for i, (k, v) in c.raw.items()}
    if c.v_own is not None:
        c.v_own = c.v_own.copy()
        c.v_own[:, :, 5] = 2.0 ** 127
        c.v_own[:, :, 6] = M.bf16(rng.uniform(-1.7e38, 1.7e38, c.v_own.shape[:2]))
        c.v_own[::5, :, c.d - 1] = -1.5 * 2.0 ** 126
    return c


FEW = ["one_key", "own_only", "empty_request", "tails", "tails_64", "pieces", "more_pieces_than_tiles", "prefill",
       "prefill_64", "cross_only", "starts", "limits", "limits_own", "limits_decode", "group_of_forty",
       "rows_80_and_6"]


@pytest.mark.parametrize("form", FEW + ROWS_256)
def test_values_as_large_as_the_format_holds(form):
    c = large(Call(form, seed=11))
    print(f"form {form}", flush=True)
    with c.store() as store:
        check(c, c.run(store))


@pytest.mark.parametrize("form", ["pieces", "decode_pieces", "decode_blocks"])
def test_every_number_of_pieces(form):
    c = large(Call(form, seed=12))
    with c.store() as store:
        for n in (1, 2, 5, 40):
            a = c.run(store, pieces=n)
            check(c, a)
            b = c.run(store, pieces=n, entry=pic.link_decode_noalloc)
            assert all(np.array_equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("form", ["tails", "rows_160_and_6", "odd_group_blocks"])
def test_one_large_value_late(form):
    """A single key with the largest value in one channel, whose score passes all before it."""
    c = Call(form, seed=13)
    for i, (k, v) in c.raw.items():
        v = v.copy()
        v[-1, :, c.d - 3] = np.inf
        c.raw[i] = (k, v)
    c.q = M.bf16(3 * c.q)
    with c.store() as store:
        check(c, c.run(store))


@pytest.mark.parametrize("form", ["tails", "rows_160_and_6", "row_limits_blocks_64"])
def test_the_reference_agrees_on_ordinary_values(form):
    c = Call(form, seed=14)
    with c.store() as store:
        check(c, c.run(store))


@pytest.mark.parametrize("form", ["own_only", "tails", "own_900", "own_900_64", "limits_own"])
def test_own_values_near_the_largest(form):
    """A channel of own values 2.6% below bf16's largest number: their means stay finite."""
    c = Call(form, seed=15)
    c.v_own = c.v_own.copy()
    c.v_own[:, :, 9] = M.bf16(3.3e38)
    c.v_own[:, :, 40] = M.bf16(np.where(np.arange(len(c.v_own)) % 2, 3.3e38, -3.3e38))[:, None]
    with c.store() as store:
        check(c, c.run(store))
