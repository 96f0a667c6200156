"""Link attention of requests that share linked chunks, against its definition in 64 bits (the
parity bar of parity_gate.py; rows merged from partials have the rounding of the split calls)."""
import itertools

import numpy as np
import pytest
import torch

import link_model as L
from paper_2602_01519_amd import pic

pytestmark = pytest.mark.gpu


class Batch:
    """A store and a batch of requests in groups. shared, mine: chunk lengths, by group and request."""

    def __init__(self, rng, kind, dtype, hkv, dk, dv, group, per, shared, mine, q_len, own=None, limits=False,
                 starts=False, layers=1):
        self.hq, self.scale = hkv * group, float(np.float32(dk ** -0.5))
        self.io = pic.BF16 if dtype == pic.FP4 else dtype
        self.mla, self.per, self.q_len, self.dv = kind == pic.MLA, per, q_len, dv
        lens = [n for l in shared + mine for n in l]
        self.store = pic.Store(kind, dtype, hkv, dk, dv, max(64, sum((n + 63) // 64 * 64 for n in lens)), n_layers=layers)
        at, cut = itertools.count(1), lambda n: 64 if starts and n > 64 else 0
        k_all, v_all = {}, {}

        def put(lists):
            out = [[next(at) for _ in l] for l in lists]
            for l, names in zip(lists, out):
                for n, i in zip(l, names):
                    k = L.draw(rng, self.io, layers, n, hkv, dk)
                    v = None if self.mla else L.draw(rng, self.io, layers, n, hkv, dv)
                    self.store.put(i, n, k, v, L.stream())
                    k_all[i], v_all[i] = [], []
                    for layer in range(layers):         # as the store holds them
                        kk = torch.empty_like(k[0])
                        vv = None if self.mla else torch.empty_like(v[0])
                        pic.debug_gather(self.store, [i], kk, vv, L.stream(), layer)
                        k_all[i].append(kk)
                        v_all[i].append(kk[..., :dv] if self.mla else vv)
            return out

        self.shared, self.mine = put(shared), put(mine)
        flat = lambda lists: [i for l in lists for i in l]  # noqa: E731
        self.groups = (L.offsets(per), L.offsets([len(l) for l in self.shared]), flat(self.shared))
        own = None if own is None else [a + b for a, b in zip(q_len, own)]
        tq = sum(q_len)
        self.q = L.draw(rng, self.io, tq, self.hq, dk)
        self.ko = None if own is None else L.draw(rng, self.io, sum(own), hkv, dk)
        self.vo = None if own is None or self.mla else L.draw(rng, self.io, sum(own), hkv, dv)
        self.args = (L.offsets([len(l) for l in self.mine]), flat(self.mine), L.offsets(q_len),
                     None if own is None else L.offsets(own), self.hq)
        start = lambda lists, lens: [cut(n) for l in lens for n in l]  # noqa: E731
        self.kw = dict(chunk_starts=start(self.mine, mine), group_starts=start(self.shared, shared)) if starts else {}
        docs = [sum(n - cut(n) for n in l) for l in mine]
        lim = [rng.integers(0, d + 1, n) for d, n in zip(docs, q_len)] if limits else None
        if limits:
            self.kw["q_doc_limits"] = np.concatenate(lim)
        self.refs = []
        for layer in range(layers):
            out, lse, r, s0 = [], [], 0, 0
            for g, n in enumerate(per):
                for r in range(r, r + n):
                    lq, ls = q_len[r], own[r] if own else 0
                    names, sizes = self.shared[g] + self.mine[r], list(shared[g]) + list(mine[r])
                    ks = [k_all[i][layer][cut(m):] for i, m in zip(names, sizes)]
                    vs = [v_all[i][layer][cut(m):] for i, m in zip(names, sizes)]
                    if ls:
                        ks.append(self.ko[s0:s0 + ls])
                        vs.append(self.ko[s0:s0 + ls, :, :dv] if self.mla else self.vo[s0:s0 + ls])
                    common = sum(m - cut(m) for m in shared[g])
                    q = self.q[self.args[2][r]:self.args[2][r + 1]]
                    seen = L.causal(lq, ls, common + docs[r], None if lim is None else lim[r] + common)
                    empty = q.new_zeros(0, hkv, dk), q.new_zeros(0, hkv, dv)
                    o, l = L.attend(q, torch.cat(ks) if ks else empty[0], torch.cat(vs) if vs else empty[1], self.scale, seen)
                    out.append(o)
                    lse.append(l)
                    s0 += ls
                r += 1 if n else 0
            self.refs.append((torch.cat(out), torch.cat(lse)))

    def buffers(self):
        out = torch.full((len(self.q), self.hq, self.dv), 7.0, dtype=self.q.dtype, device="cuda")
        return out, torch.full(self.q.shape[:2], 3.0, dtype=torch.float32, device="cuda")

    def call(self, layer=0, stream=None, out=None, lse=None):
        if out is None:
            out, lse = self.buffers()
        pic.link_shared(self.store, *self.groups, *self.args, self.q, self.ko, self.vo, self.scale, out, lse,
                        stream=L.stream() if stream is None else stream, layer=layer, **self.kw)
        return out, lse

    def plan(self):
        return pic.SharedLinkPlan(self.store, *self.groups, *self.args, **self.kw)

    def run(self, plan, layer=0, out=None, lse=None):
        if out is None:
            out, lse = self.buffers()
        plan.run(layer, self.q, self.ko, self.vo, self.scale, out, lse, L.stream())
        return out, lse

    def check(self, out, lse, layer=0, label=""):
        torch.cuda.synchronize()
        L.check(self.io, out, lse, *self.refs[layer], label)


SHAPES = [
    ("bf16-128", pic.GQA, pic.BF16, 2, 128, 128, 4), ("bf16-128-wide", pic.GQA, pic.BF16, 1, 128, 128, 8),
    ("bf16-128-odd", pic.GQA, pic.BF16, 3, 128, 128, 5), ("bf16-128-mha", pic.GQA, pic.BF16, 3, 128, 128, 1),
    ("bf16-64", pic.GQA, pic.BF16, 2, 64, 64, 3),
    ("bf16-32", pic.GQA, pic.BF16, 2, 32, 32, 4), ("f32-64", pic.GQA, pic.F32, 2, 64, 64, 4),
    ("f32-128", pic.GQA, pic.F32, 1, 128, 128, 3), ("f32-40", pic.GQA, pic.F32, 2, 40, 24, 2),
    ("bf16-96", pic.GQA, pic.BF16, 2, 96, 96, 2), ("mla", pic.MLA, pic.BF16, 1, 576, 512, 16),
    ("mla-f32", pic.MLA, pic.F32, 1, 72, 64, 3), ("bf16-512", pic.GQA, pic.BF16, 1, 64, 512, 2),
    ("fp4-128", pic.GQA, pic.FP4, 2, 128, 128, 4), ("fp4-64", pic.GQA, pic.FP4, 2, 64, 64, 3)]
KINDS = pytest.mark.parametrize("shape", SHAPES, ids=[s[0] for s in SHAPES])


@KINDS
@pytest.mark.parametrize("own", [True, False])
def test_one_token_each(shape, own):
    """Decode steps: groups of several sizes, one alone, one that shares nothing, an empty one."""
    rng = np.random.default_rng(3)
    per = [5, 1, 0, 3, 21]
    b = Batch(rng, *shape[1:], per, [[70, 64, 1], [300], [64], [], [65, 130, 500]],
              [[], [90], [1, 64], [], [3], [], [70], [], [200]] + [[]] * 19 + [[5, 6]] + [[]], [1] * 30,
              own=[int(x) for x in rng.integers(0, 140, 30)] if own else None)
    out, lse = b.call()
    b.check(out, lse, label="call")
    with b.plan() as plan:
        for _ in range(2):
            o, l = b.run(plan)
            torch.cuda.synchronize()
            assert torch.equal(o, out) and torch.equal(l, lse)


@KINDS
@pytest.mark.parametrize("limits,starts", [(False, False), (True, False), (False, True)])
def test_ragged_questions(shape, limits, starts):
    rng = np.random.default_rng(4)
    q_len = [0, 3, 17, 1, 40, 2, 0, 9]
    b = Batch(rng, *shape[1:], [3, 4, 1], [[70, 200], [64, 129, 30], [100]],
              [[90, 20], [], [130], [64], [5], [], [70], [65, 66]], q_len, own=None if limits else [2, 0, 5, 100, 0, 0, 3, 64],
              limits=limits, starts=starts)
    b.check(*b.call())
    with b.plan() as plan:
        b.check(*b.run(plan), label="plan")


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[4], SHAPES[6]], ids=lambda s: s[0])
@pytest.mark.parametrize("n", [2, 4, 5, 17, 40, 70])
def test_sizes_of_a_group(shape, n):
    """Rows of a group from one workgroup's to several, over few and many keys."""
    rng = np.random.default_rng(n)
    for shared in ([1], [64], [2500, 33]):
        b = Batch(rng, *shape[1:], [n], [shared], [[]] * n, [1] * n, own=[int(x) for x in rng.integers(0, 40, n)])
        b.check(*b.call(), label=str(shared))


@pytest.mark.parametrize("shape,q_len", [(SHAPES[0], 1), (SHAPES[0], 6), (SHAPES[1], 1), (SHAPES[3], 1), (SHAPES[4], 9)],
                         ids=lambda x: x[0] if isinstance(x, tuple) else str(x))
def test_log_sums_are_of_unrounded_probabilities(shape, q_len):
    """Few keys, where a probability rounded to bf16 would show in the log-sum-exp. Products of bf16
    elements are exact in fp32, so a logit is off by at most d_k roundings of the sum of its products'
    sizes; the sums of n probabilities, their exponents, maxima and joins by at most n + 32 more of
    numbers up to the logits' size."""
    rng = np.random.default_rng(11)
    n = 5
    b = Batch(rng, *shape[1:], [n], [[3]], [[2]] * n, [q_len] * n, own=[2] * n)
    out, lse = b.call()
    b.check(out, lse)
    d, hkv = shape[4], shape[3]
    size = 0.0
    for r in range(n):
        kk = torch.empty(5, hkv, d, dtype=torch.bfloat16, device="cuda")
        pic.debug_gather(b.store, b.shared[0] + b.mine[r], kk, torch.empty_like(kk), L.stream())
        q = b.q[r * q_len:(r + 1) * q_len].double().abs()
        k = torch.cat([kk, b.ko[r * (q_len + 2):(r + 1) * (q_len + 2)]]).double().abs()
        for h in range(b.hq):
            size = max(size, b.scale * float((q[:, h] @ k[:, h // (b.hq // hkv)].T.contiguous()).max()))
    bound = 2.0 ** -24 * (d * size + (7 + q_len + 32) * (1 + size))
    assert bound < 3e-4     # (a probability rounded to bf16 is off by up to 2 ** -8 = 4e-3 of it)
    assert float((lse.double() - b.refs[0][1]).abs().max()) <= bound


def test_long_calls():
    """More work than one launch takes: the groups' blocks and the requests' units in a launch each."""
    rng = np.random.default_rng(12)
    n = 160
    b = Batch(rng, pic.GQA, pic.BF16, 2, 128, 128, 8, [n], [[25001]], [[70]] + [[]] * (n - 1), [1] * n,
              own=[int(x) for x in rng.integers(0, 90, n)])
    b.check(*b.call())
    with b.plan() as plan:
        b.check(*b.run(plan), label="plan")


def test_rows_that_see_nothing():
    rng = np.random.default_rng(5)
    for shape in SHAPES[:1] + SHAPES[4:9]:
        b = Batch(rng, *shape[1:], [2, 1], [[], []], [[], [70], []], [1, 2, 3])
        out, lse = b.call()
        b.check(out, lse)
        assert bool((out[:1] == 0).all()) and bool(torch.isinf(lse[3:]).all())
        b = Batch(rng, *shape[1:], [1, 1], [[], []], [[], []], [2, 3])
        out, lse = b.call()
        b.check(out, lse)


def test_far_logits_and_large_values():
    """A group's rows whose logits lie far apart between the shared and the own part, and values near
    the largest of the format."""
    rng = np.random.default_rng(6)
    for shape in (SHAPES[0], SHAPES[4], SHAPES[6]):
        b = Batch(rng, *shape[1:], [6], [[130, 70]], [[30]] * 6, [1] * 6, own=[3] * 6)
        b.q *= 60.0
        d = shape[4]
        b.ko *= torch.where(torch.arange(len(b.ko), device="cuda") % 2 == 0, 50.0, -50.0)[:, None, None].to(b.ko.dtype)
        out, lse = b.call()
        torch.cuda.synchronize()
        # the reference again, with the tensors as they are now
        k, v = torch.empty(200, shape[3], d, dtype=b.q.dtype, device="cuda"), torch.empty(200, shape[3], d, dtype=b.q.dtype, device="cuda")
        pic.debug_gather(b.store, b.shared[0], k, v, L.stream())
        for r in range(6):
            mk, mv = torch.empty(30, shape[3], d, dtype=k.dtype, device="cuda"), torch.empty(30, shape[3], d, dtype=k.dtype, device="cuda")
            pic.debug_gather(b.store, b.mine[r], mk, mv, L.stream())
            o, l = L.attend(b.q[r:r + 1], torch.cat([k, mk, b.ko[4 * r:4 * r + 4]]), torch.cat([v, mv, b.vo[4 * r:4 * r + 4]]), b.scale)
            # logits of thousands: fp32 products round them by 2^-22 of their size each
            assert float((lse[r] - l[0]).abs().max()) <= 4e-3 + 2.0 ** -20 * float(l.abs().max())
            near = (lse[r].double() - l[0]).abs() < 1e-3
            assert bool(torch.isfinite(out[r]).all()) and near.any()


@pytest.mark.parametrize("q_len,per", [(9, 2), (3, 2), (40, 3), (1, 3)])
def test_values_near_the_largest(q_len, per):
    """64-wide heads: values up to 2^126 under logits that rise by 40 along the keys, so that unnormalised
    sums would leave the fp32 range. (Up to 16 rows run the streaming kernel, whose probabilities go up to
    one: some 13 of them here, which takes 2^126 out of the range in it as in every link call of
    64-wide heads. There the values go up to 2^101.) A probability is off by half a bf16 step, 2^-8 of it, the
    logits (exact products of 8 and at most 40) and fp32 sums by less than 2^-12, the output by half a step."""
    rng = np.random.default_rng(15)
    n = per
    b = Batch(rng, pic.GQA, pic.BF16, 2, 64, 64, 4, [n], [[]], [[]] * n, [q_len] * n, own=[30] * n)
    store = pic.Store(pic.GQA, pic.BF16, 2, 64, 64, 64 * 30)
    big = lambda *s: (L.draw(rng, pic.F32, *s).clamp(-2, 2) * 2.0 ** (125 if q_len > 4 else 100)).bfloat16()  # noqa: E731
    lens = [700, 130]

    def rising(m, lo, hi):
        k = torch.zeros(m, 2, 64, dtype=torch.bfloat16, device="cuda")
        k[:, :, 0] = torch.linspace(lo, hi, m, device="cuda").bfloat16()[:, None]
        return k

    ks, vs = [rising(700, 0, 30), rising(130, 30, 40)], [big(m, 2, 64) for m in lens]
    for i, m in enumerate(lens):
        store.put(1 + i, m, ks[i], vs[i], L.stream())
    own = q_len + 30
    q = torch.zeros(n * q_len, 8, 64, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 8.0                            # (the scale is 1 / 8)
    ko, vo = torch.cat([rising(own, 0, 40) for _ in range(n)]), big(n * own, 2, 64)
    out, lse = torch.empty_like(q), torch.empty(n * q_len, 8, dtype=torch.float32, device="cuda")
    pic.link_shared(store, [0, n], [0, 2], [1, 2], [0] * (n + 1), [], L.offsets([q_len] * n), L.offsets([own] * n), 8, q, ko,
                    vo, b.scale, out, lse, stream=L.stream())
    torch.cuda.synchronize()
    for r in range(n):
        at, rows = slice(r * q_len, (r + 1) * q_len), slice(r * own, (r + 1) * own)
        k, v = torch.cat(ks + [ko[rows]]), torch.cat(vs + [vo[rows]])
        seen = L.causal(q_len, own, 830)
        ref, ref_lse = L.attend(q[at], k, v, b.scale, seen)
        size, _ = L.attend(q[at], k, v.abs(), b.scale, seen)
        # (single tokens: sums of rounded probabilities, off by as much again)
        bound = size * ((2.0 if q_len == 1 else 1.0) * 2.0 ** -8 + 2.0 ** -11) + ref.abs() * 2.0 ** -8
        assert bool(torch.isfinite(out[at]).all())
        assert bool(((out[at].double() - ref).abs() <= bound).all())
        assert float((lse[at].double() - ref_lse).abs().max()) <= 2.0 ** -8 + 2.0 ** -11


def test_layers_streams_and_graphs():
    rng = np.random.default_rng(7)
    b = Batch(rng, pic.GQA, pic.BF16, 2, 128, 128, 4, [6, 3], [[300, 65], [130]], [[20]] + [[]] * 8, [1] * 9,
              own=[int(x) for x in rng.integers(0, 100, 9)], layers=3)
    for layer in range(3):
        b.check(*b.call(layer), layer, "call")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [b.buffers() for _ in range(6)]
    torch.cuda.synchronize()
    for i, (o, l) in enumerate(outs):           # several in flight, on two streams
        b.call(i % 3, side.cuda_stream if i % 2 else L.stream(), o, l)
    side.synchronize()
    for i, (o, l) in enumerate(outs):
        b.check(o, l, i % 3, "two streams")
    with b.plan() as plan, b.plan() as other:
        graphs = []
        for i, p in enumerate((plan, other, plan)):
            o, l = b.buffers()
            g = torch.cuda.CUDAGraph()
            b.run(p, i, o, l)
            with torch.cuda.graph(g):
                b.run(p, i, o, l)
            graphs.append((g, o, l))
        for _ in range(3):
            for i, (g, o, l) in enumerate(graphs):
                o.fill_(2.0)
                g.replay()
                b.check(o, l, i, "graph")
            b.check(*b.call(1), 1, "between replays")
        with pytest.raises(pic.PicError):       # the plans hold shared chunks and own ones alike
            b.store.remove(b.shared[0][0], L.stream())
        with pytest.raises(pic.PicError):
            b.store.remove(b.mine[0][0], L.stream())
    b.store.remove(b.shared[0][0], L.stream())
    b.store.remove(b.mine[0][0], L.stream())


@pytest.mark.parametrize("own", [True, False])
def test_narrow_heads_by_layer_captured(own):
    """64-wide heads, several tokens: groups' and requests' blocks in one launch, own KV laid out before it."""
    rng = np.random.default_rng(16)
    q_len = [9, 1, 40, 0, 5]
    b = Batch(rng, pic.GQA, pic.BF16, 2, 64, 64, 4, [3, 2], [[300, 65], [130]], [[20], [], [70, 1], [], []], q_len,
              own=[3, 0, 64, 2, 0] if own else None, layers=2)
    with b.plan() as plan, b.plan() as other:
        graphs = []
        for p, layer in ((plan, 0), (other, 1), (plan, 1)):
            out, lse = b.buffers()
            b.run(p, layer, out, lse)
            b.check(out, lse, layer, "run")
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                b.run(p, layer, out, lse)
            graphs.append((g, out, lse, layer))
        for _ in range(3):
            for g, out, lse, layer in graphs:
                out.fill_(2.0)
                g.replay()
                b.check(out, lse, layer, "graph")
            b.check(*b.call(1), 1, "between replays")


def test_a_capture_takes_plans_alone():
    rng = np.random.default_rng(13)
    b = Batch(rng, pic.GQA, pic.BF16, 2, 128, 128, 4, [6], [[300]], [[]] * 6, [1] * 6, own=[9] * 6)
    out, lse = b.buffers()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(pic.PicError) as e:
            b.call(out=out, lse=lse)
        assert e.value.status == pic.ERR_UNSUPPORTED
        b.q.add_(0)
    torch.cuda.synchronize()
    assert bool((out == 7).all())
    b.check(*b.call())


def test_growing_chunks_behind_shared_documents():
    """Decode steps whose own tokens live in growing chunks, behind the group's documents."""
    rng = np.random.default_rng(8)
    b = Batch(rng, pic.GQA, pic.BF16, 2, 128, 128, 4, [4], [[200, 70]], [[]] * 4, [1] * 4)
    store = pic.Store(pic.GQA, pic.BF16, 2, 128, 128, 64 * 20)
    kc, vc = (L.draw(rng, pic.BF16, 270, 2, 128) for _ in range(2))
    store.put(1, 270, kc, vc, L.stream())
    for r in range(4):
        store.open(10 + r, 130)
    held = [[], [], [], []]
    with pic.Rope(pic.BF16, pic.ROPE_HALF, 128, 0, 128) as rope:
        for step in range(5):
            n = [1, 30 * (step == 0) + 1, 1, 63 if step == 0 else 1]
            at = L.offsets(n)
            k, v = (L.draw(rng, pic.BF16, sum(n), 2, 128) for _ in range(2))
            pos = torch.arange(sum(n), dtype=torch.int32, device="cuda") + 270
            store.append([10 + r for r in range(4)], at, k, v, rope, pos, stream=L.stream())
            q = L.draw(rng, pic.BF16, 4, 8, 128)
            out, lse = torch.empty_like(q), torch.empty(4, 8, dtype=torch.float32, device="cuda")
            pic.link_shared(store, [0, 4], [0, 1], [1], range(5), [10 + r for r in range(4)], range(5), None, 8, q, None,
                            None, b.scale, out, lse, stream=L.stream())
            torch.cuda.synchronize()
            for r in range(4):
                held[r].append(v[at[r]:at[r + 1]])
                m = sum(len(x) for x in held[r])
                kk, vv = (torch.empty(270 + m, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
                pic.debug_gather(store, [1, 10 + r], kk, vv, L.stream())
                assert torch.equal(vv, torch.cat([vc] + held[r]))
                L.check(pic.BF16, out[r:r + 1], lse[r:r + 1], *L.attend(q[r:r + 1], kk, vv, b.scale))


def test_refusals_write_nothing():
    rng = np.random.default_rng(9)
    b = Batch(rng, pic.GQA, pic.BF16, 1, 128, 128, 2, [2, 1], [[70], [64]], [[5], [], []], [1, 1, 1], own=[0, 0, 0])
    g, a = [np.array(x) for x in b.groups], list(b.args)
    ids = g[2].astype(np.uint64)
    out, lse = b.buffers()

    def bad(status, groups=None, args=None, scale=b.scale, q=b.q, ko=b.ko, **kw):
        with pytest.raises(pic.PicError) as e:
            pic.link_shared(b.store, *(groups or g), *(args or a), q, ko, b.vo, scale, out, lse, stream=L.stream(), **kw)
        assert e.value.status == status, (groups, args, kw)

    INV = pic.ERR_INVALID
    bad(INV, groups=[[0, 2, 4], g[1], ids])
    bad(INV, groups=[[0, 3, 2], g[1], ids])
    bad(INV, groups=[[1, 2, 3], g[1], ids])
    bad(INV, groups=[g[0], [0, 2, 1], ids])
    bad(INV, groups=[[0, 2], [0, 1], ids])
    bad(pic.ERR_NOT_FOUND, groups=[g[0], g[1], [ids[0], 99]])
    bad(INV, group_starts=[64, 64])
    bad(INV, group_starts=[1, 0])
    bad(INV, args=a[:4] + [3 * 7 + 2 ** 30])
    bad(INV, args=[a[0], a[1], [0, 1, 2, 1], a[3], a[4]])
    bad(INV, scale=float("nan"))
    bad(INV, q=None)
    bad(INV, ko=None)
    bad(INV, layer=1)
    bad(INV, q_doc_limits=[6, 0, 0])
    with pytest.raises(pic.PicError):
        pic.SharedLinkPlan(b.store, [0, 2], [0, 1], ids[:1], *a)
    with pytest.raises(pic.PicError) as e:       # more output rows of a request than a launch merges
        pic.SharedLinkPlan(b.store, [0, 1], [0, 1], ids[:1], [0, 0], [], [0, 2 ** 25], None, 2)
    assert e.value.status == pic.ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and bool((lse == 3).all())
    # nothing to do
    pic.link_shared(b.store, [0], [0], [], [0], [], [0], None, 2, None, None, None, 1.0, None)
    with pic.SharedLinkPlan(b.store, [0], [0], [], [0], [], [0], None, 2) as plan:
        plan.run(0, None, None, None, 1.0, None)
