"""Link attention over selected blocks against its definition in 64 bits: the taken blocks exactly,
outputs by the parity bar of parity_gate.py."""
import numpy as np
import pytest
import torch

import link_model as L
from paper_2602_01519_amd import pic

pytestmark = pytest.mark.gpu


def summaries(k, sizes):
    """Means of the 64-token blocks of the links (sizes tokens each) of keys k [tokens][heads][d]."""
    means, block, at = [], [], 0
    for n in sizes:
        for b in range(0, n, 64):
            m = min(64, n - b)
            block += [len(means)] * m
            means.append((k[at + b:at + b + m].double().sum(0) / m).float().to(torch.bfloat16).double())
        at += n
    return torch.stack(means), torch.tensor(block, device="cuda")


def chosen(means, q, n_blocks, first, last):
    """Blocks of one query token q [group][d] by the summaries of its kv head [blocks][d]."""
    score = (q.double() @ means.T.contiguous()).cpu().numpy()
    score = np.where(np.isnan(score), -np.inf, score).max(0)
    n = len(score)
    order = sorted(range(n), key=lambda b: (not (b < first or b >= n - last), 0.0 if b < first or b >= n - last else -score[b], b))
    return sorted(order[:n_blocks])


class Case:
    def __init__(self, rng, dtype, hkv, d, group, chunks, links, q_len, own=None, starts=False, layers=1, capacity=None):
        self.dtype, self.hkv, self.d, self.hq = dtype, hkv, d, hkv * group
        self.scale = float(np.float32(d ** -0.5))
        self.store = pic.Store(pic.GQA, dtype, hkv, d, d, capacity or 256 + sum((n + 63) // 64 * 64 for n in chunks), n_layers=layers)
        self.layers = layers
        for i, n in enumerate(chunks):
            self.put(rng, i, n)
        self.links, self.q_len = links, q_len
        self.own = None if own is None else [a + b for a, b in zip(q_len, own)]
        self.q = L.draw(rng, dtype, sum(q_len), self.hq, d)
        self.ko, self.vo = (None, None) if own is None else (L.draw(rng, dtype, sum(self.own), hkv, d) for _ in range(2))
        self.starts = [[64 if starts and i % 2 and chunks[i] > 64 else 0 for i in l] for l in links]
        self.index = pic.BlockIndex(self.store)
        self.index.update(range(len(chunks)), stream=L.stream())

    def put(self, rng, i, n):
        self.store.put(i, n, *(L.draw(rng, self.dtype, self.layers, n, self.hkv, self.d) for _ in range(2)), L.stream())

    def args(self):
        return (L.offsets([len(l) for l in self.links]), [i for l in self.links for i in l], L.offsets(self.q_len),
                None if self.own is None else L.offsets(self.own), self.hq)

    def buffers(self, n_blocks):
        return (torch.full_like(self.q, 7.0), torch.full(self.q.shape[:2], 3.0, dtype=torch.float32, device="cuda"),
                torch.full((len(self.q), self.hkv, n_blocks), -9, dtype=torch.int32, device="cuda"))

    def call(self, n_blocks, first=0, last=0, layer=0, bufs=None, stream=None):
        out, lse, blocks = bufs or self.buffers(n_blocks)
        pic.link_sparse(self.index, *self.args(), n_blocks, self.q, self.ko, self.vo, self.scale, out, lse, keep_first=first,
                        keep_last=last, blocks=blocks, stream=L.stream() if stream is None else stream, layer=layer,
                        chunk_starts=[s for l in self.starts for s in l])
        return out, lse, blocks

    def check(self, got, n_blocks, first=0, last=0, layer=0, rows=None):
        out, lse, blocks = got
        torch.cuda.synchronize()
        refs, t, s0 = [], 0, 0
        for r, l in enumerate(self.links):
            lq, ls = self.q_len[r], self.own[r] if self.own else 0
            sizes = [self.store.lookup(i) for i in l]
            k, v = (torch.empty(sum(sizes), self.hkv, self.d, dtype=self.q.dtype, device="cuda") for _ in range(2))
            pic.debug_gather(self.store, l, k, v, L.stream(), layer)
            torch.cuda.synchronize()
            kept = torch.cat([torch.arange(n, device="cuda") >= s for n, s in zip(sizes, self.starts[r])]) if l else None
            if l:
                k, v = k[kept], v[kept]
            sizes = [n - s for n, s in zip(sizes, self.starts[r])]
            if len(k):
                means, block = summaries(k, sizes)
            for i in range(lq):
                seen = torch.zeros(self.hkv, len(k), dtype=torch.bool, device="cuda")
                for h in range(self.hkv):
                    want = []
                    if len(k):
                        g = self.hq // self.hkv
                        want = chosen(means[:, h], self.q[t, h * g:(h + 1) * g], n_blocks, first, last)
                        seen[h] = torch.isin(block, torch.tensor(want, device="cuda"))
                    have = blocks[t, h].tolist()
                    assert have == want + [-1] * (n_blocks - len(want)), (r, i, h)
                g = self.hq // self.hkv
                own = slice(s0, s0 + max(0, ls - lq + i + 1) if ls else s0)
                o, z = [], []
                for h in range(self.hkv):
                    kk, vv = k[seen[h], h:h + 1], v[seen[h], h:h + 1]
                    if ls:
                        kk, vv = torch.cat([kk, self.ko[own, h:h + 1]]), torch.cat([vv, self.vo[own, h:h + 1]])
                    a, b = L.attend(self.q[t:t + 1, h * g:(h + 1) * g], kk, vv, self.scale)
                    o.append(a)
                    z.append(b)
                refs.append((torch.cat(o, 1), torch.cat(z, 1)))
                t += 1
            s0 += ls
        ref, ref_lse = (torch.cat([x[i] for x in refs]) for i in range(2))
        rows = slice(None) if rows is None else rows
        L.check(self.dtype, out[rows], lse[rows], ref[rows], ref_lse[rows], f"{n_blocks} blocks")


CHUNKS = [70, 64, 1, 300, 1000, 129, 63, 640]
LINKS = [[0, 3], [4], [], [2], [7, 0, 5, 1], [4, 4, 6]]


@pytest.mark.parametrize("dtype", [pic.BF16, pic.F32])
@pytest.mark.parametrize("hkv,d,group", [(2, 128, 4), (3, 64, 1), (1, 64, 5), (2, 64, 8), (1, 128, 20), (8, 128, 2)])
def test_shapes_and_numbers_of_blocks(dtype, hkv, d, group):
    rng = np.random.default_rng(hkv * d + group)
    c = Case(rng, dtype, hkv, d, group, CHUNKS, LINKS, [1, 2, 1, 3, 0, 1], own=[0, 70, 5, 0, 3, 200], starts=group == 4)
    for n, first, last in ((1, 0, 0), (3, 1, 1), (7, 0, 2), (4, 4, 0), (16, 3, 5), (700, 0, 0)):
        c.check(c.call(n, first, last), n, first, last)
    c.own = c.ko = c.vo = None
    for n, first, last in ((2, 0, 0), (9, 1, 0)):
        c.check(c.call(n, first, last), n, first, last)


@pytest.mark.parametrize("dtype,d", [(pic.BF16, 128), (pic.F32, 64), (pic.F32, 128), (pic.BF16, 64)])
@pytest.mark.parametrize("n", [17, 64, 129, 333])
def test_few_requests_many_blocks(dtype, d, n):
    """Units that several workgroups share, blocks past a histogram's round."""
    rng = np.random.default_rng(n)
    c = Case(rng, dtype, 1, d, 3, [30001, 4097, 64 * 700], [[0, 1], [2]], [1, 2], own=[33, 5])
    got = c.call(n, 2, 3)
    c.check(got, n, 2, 3)
    for _ in range(2):
        again = c.call(n, 2, 3)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_a_batch_larger_than_the_gpu():
    rng = np.random.default_rng(3)
    B = 150
    c = Case(rng, pic.BF16, 4, 128, 4, [int(x) for x in rng.integers(1, 900, 40)],
             [[int(x) for x in rng.integers(0, 40, rng.integers(0, 6))] for _ in range(B)], [1] * B,
             own=[int(x) for x in rng.integers(0, 90, B)])
    c.check(c.call(9, 1, 1), 9, 1, 1)


@pytest.mark.parametrize("d", [64, 128])
def test_log_sums_are_of_unrounded_probabilities(d):
    """Few keys, where a probability rounded to bf16 would show in the log-sum-exp. A logit is off by
    at most d roundings of the sum of its products' sizes, the sums of the probabilities, their
    exponents, maxima and joins by at most n + 32 more of numbers up to the logits' size."""
    rng = np.random.default_rng(12)
    c = Case(rng, pic.BF16, 2, d, 4, [3, 2, 4], [[0], [1, 0], [2]], [1, 1, 2], own=[0, 2, 1])
    got = c.call(2)
    c.check(got, 2)
    size = 0.0
    at = 0
    for r, l in enumerate(c.links):
        for i in range(c.q_len[r]):
            s0 = sum(c.own[:r])
            k = torch.empty(sum(c.store.lookup(j) for j in l), 2, d, dtype=torch.bfloat16, device="cuda")
            pic.debug_gather(c.store, l, k, torch.empty_like(k), L.stream())
            k = torch.cat([k, c.ko[s0:s0 + c.own[r] - c.q_len[r] + i + 1]]).double()
            for h in range(c.hq):
                s = c.scale * (c.q[at, h].double() * k[:, h // 4])
                size = max(size, float(s.abs().sum(1).max()))
                bound = 2.0 ** -24 * (d * size + 45 * (1 + size))
                assert bound < 3e-4
                assert abs(float(got[1][at, h]) - float(torch.logsumexp(s.sum(1), 0))) <= bound
            at += 1


@pytest.mark.parametrize("dtype,d", [(pic.BF16, 128), (pic.BF16, 64), (pic.F32, 128), (pic.F32, 64)])
def test_values_near_the_largest(dtype, d):
    """Values up to 2^126 under some 900 keys of like scores: their means stay finite. A probability is off
    by half a bf16 step, 2^-8 of it, logits and fp32 sums (128 products, 900 values) by less than 2^-11 of
    what they make, the output by half a step."""
    rng = np.random.default_rng(15)
    c = Case(rng, dtype, 2, d, 4, [70], [[0], [0]], [1, 1], own=[60, 0], capacity=64 * 40)
    k = L.draw(rng, dtype, 1, 830, 2, d) * 0.25
    big = lambda *s: (L.draw(rng, pic.F32, *s).clamp(-2, 2) * 2.0 ** 125).to(k.dtype)  # noqa: E731
    v = big(1, 830, 2, d)
    c.store.put(50, 830, k, v, L.stream())
    c.index.update([50], stream=L.stream())
    c.links = [[50], [50]]
    c.vo = big(*c.vo.shape)
    out, lse, _ = c.call(20)
    torch.cuda.synchronize()
    step = 2.0 ** -8 if dtype == pic.BF16 else 0.0
    for t, own in ((0, slice(0, 61)), (1, slice(61, 62))):
        kk, vv = torch.cat([k[0], c.ko[own]]), torch.cat([v[0], c.vo[own]])
        ref, ref_lse = L.attend(c.q[t:t + 1], kk, vv, c.scale)
        size, _ = L.attend(c.q[t:t + 1], kk, vv.abs(), c.scale)
        assert bool(torch.isfinite(out[t]).all())
        assert bool(((out[t].double() - ref[0]).abs() <= size[0] * (step + 2.0 ** -11) + ref[0].abs() * step).all())
        assert float((lse[t].double() - ref_lse[0]).abs().max()) <= 2.0 ** -11


def test_equal_scores_go_to_the_lower_block():
    rng = np.random.default_rng(4)
    c = Case(rng, pic.BF16, 2, 64, 3, [64, 128, 64], [[0, 0, 1, 0, 2, 0, 1, 0], [0] * 40], [1, 1])
    k = torch.zeros(1, 64, 2, 64, dtype=torch.bfloat16, device="cuda")
    c.store.put(50, 64, k, k, L.stream())           # zero keys: scores of 0, of either sign
    c.index.update([50], stream=L.stream())
    c.links.append([50, 50, 0, 50, 50])
    c.starts.append([0] * 5)
    c.q = torch.cat([c.q, -c.q[:1]])
    c.q_len.append(1)
    for n in (1, 2, 3, 5, 7, 13):
        c.check(c.call(n), n)
        if n < 13:
            c.check(c.call(n, 0, 1), n, 0, 1)


def test_not_a_number_and_infinities():
    rng = np.random.default_rng(5)
    c = Case(rng, pic.BF16, 1, 64, 2, [64] * 10, [list(range(10))] * 3, [1] * 3)
    bad = torch.zeros(64, 1, 64, dtype=torch.bfloat16, device="cuda")
    bad[5] = float("nan")
    c.store.put(90, 64, bad, bad, L.stream())
    c.index.update([90], stream=L.stream())
    c.links = [[90] + list(range(10)), list(range(5)) + [90] + list(range(5, 10)), list(range(10)) + [90]]
    c.starts = [[0] * 11] * 3
    got = c.call(4)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(got[0]).all())       # a block of NaN scores -inf and is not taken
    c.check(got, 4)
    c.q[1] = float("nan")                           # every score -inf: the lowest blocks
    got = c.call(4)
    torch.cuda.synchronize()
    assert got[2][1, 0].tolist() == [0, 1, 2, 3] and bool(torch.isfinite(got[0][[0, 2]]).all())


def test_what_a_change_leaves_out_of_date():
    rng = np.random.default_rng(6)
    c = Case(rng, pic.BF16, 2, 64, 2, [200, 300, 100], [[0, 1]], [1], own=[4], layers=2, capacity=64 * 40)

    def stale(layer=0):
        with pytest.raises(pic.PicError) as e:
            c.call(3, layer=layer)
        assert e.value.status == pic.ERR_INVALID

    c.check(c.call(3), 3)
    c.store.remove(1, L.stream())
    torch.cuda.synchronize()
    c.put(rng, 1, 300)
    stale()
    c.index.update([1], layer=1, stream=L.stream())
    stale(0)
    c.check(c.call(3, layer=1), 3, layer=1)
    c.index.update([1, 1], stream=L.stream())
    c.check(c.call(3), 3)
    # a derived chunk, then rows written into it
    c.store.derive(7, 0, [70, 130], L.stream())
    c.links = [[7, 1, 2]]
    c.starts = [[0] * 3]
    stale()
    c.index.update([7], stream=L.stream())
    c.check(c.call(5), 5)
    k, v = (L.draw(rng, pic.BF16, 2, 2, 64) * 9 for _ in range(2))
    c.store.write_rows(7, 1, [70, 130], k, v, L.stream())
    stale(1)
    c.index.update([7], stream=L.stream())
    for layer in range(2):
        c.check(c.call(5, layer=layer), 5, layer=layer)
    # a chunk that grows: each step's blocks formed again as far as they grew
    c.store.open(8, 400)
    c.links = [[8, 2]]
    c.starts = [[0, 0]]
    c.index.update([8], stream=L.stream())
    c.check(c.call(2), 2)
    for n in (1, 62, 1, 1, 130, 64, 3):
        for layer in range(2):
            c.store.append([8], [0, n], *(L.draw(rng, pic.BF16, n, 2, 64) for _ in range(2)), stream=L.stream(), layer=layer)
        stale()
        c.index.update([8], stream=L.stream())
        for layer in range(2):
            c.check(c.call(3, 0, 1, layer=layer), 3, 0, 1, layer=layer)
    c.store.truncate([8], [100], L.stream())
    stale()
    c.index.update([8], stream=L.stream())
    c.check(c.call(3), 3)
    c.store.truncate([8], [100], L.stream())        # nothing taken back
    c.check(c.call(3), 3)
    # layers that hold differently many tokens
    c.store.append([8], [0, 5], *(L.draw(rng, pic.BF16, 5, 2, 64) for _ in range(2)), stream=L.stream(), layer=1)
    stale(1)
    c.check(c.call(3), 3)
    c.index.update([8], stream=L.stream())
    c.check(c.call(3), 3)
    c.call(3, layer=1)


def test_blocks_of_scattered_runs():
    rng = np.random.default_rng(7)
    c = Case(rng, pic.F32, 1, 64, 2, [64] * 30, [[]], [2], capacity=64 * 30)
    for i in (1, 4, 5, 6, 11, 13, 14, 20, 22, 29):
        c.store.remove(i, L.stream())
    torch.cuda.synchronize()
    c.put(rng, 40, 640 - 7)
    c.index.update([40], stream=L.stream())
    c.links, c.starts = [[0, 40, 2]], [[0, 64, 0]]
    for n in (1, 4, 11, 12):
        c.check(c.call(n, 0, 1), n, 0, 1)


def test_many_heads():
    """The most kv heads, and more chunks than one launch of summaries takes."""
    rng = np.random.default_rng(14)
    c = Case(rng, pic.BF16, 256, 64, 1, [70, 1, 130] + [5] * 100, [[0, 1], [2, 102]], [1, 1], own=[3, 0])
    c.check(c.call(2, 0, 1), 2, 0, 1)


@pytest.mark.parametrize("blocks,ok", [(8192, True), (8193, False)])
def test_longest_requests(blocks, ok):
    rng = np.random.default_rng(8)
    n = blocks * 64 - 5
    with pic.Store(pic.GQA, pic.BF16, 1, 64, 64, blocks * 64) as store:
        k = torch.randn(n, 1, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
        store.put(1, n, k, k, L.stream())
        with pic.BlockIndex(store) as index:
            index.update([1], stream=L.stream())
            q = L.draw(rng, pic.BF16, 1, 2, 64)
            out, lse = torch.full_like(q, 7.0), torch.zeros(1, 2, dtype=torch.float32, device="cuda")
            taken = torch.full((1, 1, 1024), -9, dtype=torch.int32, device="cuda")
            call = lambda m: pic.link_sparse(index, [0, 1], [1], [0, 1], None, 2, m, q, None, None, 0.125, out, lse,  # noqa: E731
                                             keep_first=1, keep_last=1, blocks=taken, stream=L.stream())
            if not ok:
                with pytest.raises(pic.PicError) as e:
                    call(1024)
                assert e.value.status == pic.ERR_UNSUPPORTED
                return
            means = torch.stack([x.double().mean(0) for x in k[:, 0].split(64)]).float().bfloat16().double()
            for m in (1024, 40, 2):
                call(m)
                torch.cuda.synchronize()
                want = chosen(means, q[0], m, 1, 1)
                assert taken.flatten()[:m].tolist() == want
                rows = torch.cat([torch.arange(b * 64, min(n, b * 64 + 64)) for b in want]).cuda()
                L.check(pic.BF16, out, lse, *L.attend(q, k[rows], k[rows], 0.125), str(m))
            with pytest.raises(pic.PicError):
                call(1025)


def test_streams_layers_and_graphs():
    rng = np.random.default_rng(9)
    c = Case(rng, pic.BF16, 2, 128, 4, [700, 300, 64, 900], [[0, 1], [2, 3], [3]], [1, 1, 2], own=[9, 0, 70], layers=3)
    big = Case(rng, pic.BF16, 2, 128, 4, [700, 300, 64, 900], [[0, 1], [2, 3], [3]] * 30, [1] * 90, own=[9] * 90)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    bufs = [(c if i % 3 else big).buffers(5) for i in range(9)]
    torch.cuda.synchronize()
    for i, b in enumerate(bufs):
        (c if i % 3 else big).call(5, 1, 0, layer=i % 3 and i % 2, bufs=b, stream=side.cuda_stream if i % 2 else L.stream())
    side.synchronize()
    for i, b in enumerate(bufs):
        (c if i % 3 else big).check(b, 5, 1, 0, layer=i % 3 and i % 2)
    # a small call, its tables a kernel argument, captured: replayed with new queries
    graphs = []
    for layer in (0, 2):
        b = c.buffers(5)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call(5, 0, 1, layer=layer, bufs=b)
        graphs.append((g, b, layer))
    for _ in range(3):
        c.q.copy_(L.draw(rng, pic.BF16, *c.q.shape))
        for g, b, layer in graphs:
            g.replay()
            c.check(b, 5, 0, 1, layer)
        c.check(c.call(4), 4)


def test_captured_calls():
    """A capture takes no memory of the store's: a unit that eager calls share out is one workgroup's."""
    rng = np.random.default_rng(13)
    c = Case(rng, pic.BF16, 2, 128, 4, [700, 300, 64, 900], [[0, 1, 2, 3, 0, 3]], [1], own=[40])
    bufs, g = c.buffers(24), torch.cuda.CUDAGraph()
    c.check(c.call(24, 1, 1), 24, 1, 1)
    with torch.cuda.graph(g):
        c.call(24, 1, 1, bufs=bufs)
    for _ in range(3):
        c.q.copy_(L.draw(rng, pic.BF16, *c.q.shape))
        eager = [c.call(24, 1, 1) for _ in range(9)]        # (every workspace of the store)
        g.replay()
        c.check(bufs, 24, 1, 1)
        for x in eager:
            c.check(x, 24, 1, 1)
    c.links, c.starts = [[0] * 89], [[0] * 89]
    out = c.buffers(24)
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(pic.PicError) as e:
            c.call(24, bufs=out)
        assert e.value.status == pic.ERR_UNSUPPORTED
        c.q.add_(0)
    torch.cuda.synchronize()
    assert bool((out[0] == 7).all())
    c.check(c.call(24), 24)


def test_refusals_write_nothing():
    rng = np.random.default_rng(10)
    c = Case(rng, pic.BF16, 2, 64, 2, [200, 300], [[0, 1]], [1], own=[4])
    bufs = c.buffers(4)
    a = list(c.args())

    def bad(status, n=4, args=None, scale=c.scale, q=c.q, ko=c.ko, **kw):
        with pytest.raises(pic.PicError) as e:
            pic.link_sparse(c.index, *(args or a), n, q, ko, c.vo, scale, bufs[0], bufs[1], blocks=bufs[2], stream=L.stream(), **kw)
        assert e.value.status == status, kw

    INV = pic.ERR_INVALID
    bad(INV, n=0)
    bad(INV, n=-3)
    bad(pic.ERR_UNSUPPORTED, n=1025)
    bad(INV, keep_first=3, keep_last=2)
    bad(INV, keep_first=-1)
    bad(INV, keep_last=-1)
    bad(INV, keep_first=2 ** 31 - 1, keep_last=2 ** 31 - 1)
    bad(INV, layer=1)
    bad(INV, layer=-1)
    bad(INV, scale=0.0)
    bad(INV, q=None)
    bad(INV, ko=None)
    bad(INV, chunk_starts=[0, 320])
    bad(INV, args=a[:4] + [3])
    bad(pic.ERR_NOT_FOUND, args=[a[0], [0, 5], *a[2:]])
    torch.cuda.synchronize()
    assert bool((bufs[0] == 7).all()) and bool((bufs[1] == 3).all()) and bool((bufs[2] == -9).all())
    for call, status in ((lambda: c.index.update([0], layer=1), INV), (lambda: c.index.update([0], layer=-2), INV),
                         (lambda: c.index.update([0, 9]), pic.ERR_NOT_FOUND), (lambda: c.store.close(), INV)):
        with pytest.raises(pic.PicError) as e:
            call()
        assert e.value.status == status
    for desc in ((pic.GQA, pic.FP4, 2, 64, 64), (pic.MLA, pic.BF16, 1, 576, 512), (pic.GQA, pic.BF16, 2, 32, 32),
                 (pic.GQA, pic.F32, 2, 64, 128)):
        with pytest.raises(pic.PicError) as e:
            pic.BlockIndex(pic.Store(*desc, 64))
        assert e.value.status == pic.ERR_UNSUPPORTED
    # nothing to do
    pic.link_sparse(c.index, [0], [], [0], None, 4, 3, None, None, None, 1.0, None)
    c.index.update([], stream=L.stream())
    c.index.close()
    with pytest.raises(pic.PicError):
        c.index.update([0])
    c.store.close()
