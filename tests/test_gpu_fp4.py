"""Stores that hold their chunk caches in 4 bits, and link attention over them, against the
definition in 64 bits (fp4_model.py, which derives the tolerances)."""
import numpy as np
import pytest
import torch

import fp4_model as M
from paper_2602_01519_amd import pic

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def dev(x, shift=0):
    """bf16 values on the GPU; shift: elements between an aligned address and the first."""
    b = M.bits(x)
    t = torch.zeros(b.size + shift, dtype=torch.int16, device="cuda")
    t[shift:] = torch.from_numpy(b.reshape(-1)).cuda()
    return t[shift:].view(*b.shape)


def host(t):
    u = t.cpu().numpy().view(np.uint16).astype(np.uint32) << 16
    return u.view(np.float32).astype(np.float64)


def gather(store, ids, n, hkv, d, layer=0):
    k = torch.full((n, hkv, d), 77, dtype=torch.int16, device="cuda")
    v = torch.full((n, hkv, d), 77, dtype=torch.int16, device="cuda")
    pic.debug_gather(store, ids, k, v, stream(), layer=layer)
    torch.cuda.synchronize()
    return host(k), host(v)


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def wild(rng, shape):
    """Blocks of very different sizes, zeros, values on the borders between two codes."""
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-30, 30, shape[:-1] + (1,))
    b = x.reshape(-1, 32)
    kind = rng.integers(0, 8, len(b))
    b[kind == 0] = 0
    edge = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 6.5, 6.96875, 7, 0.5, 1, 3, 4, -7])
    b[kind == 1, :16] = edge
    b[kind == 1, 16:] = -edge
    b[kind == 2, 16:] *= 2.0 ** -12
    b[kind == 3] = np.sign(b[kind == 3]) * 2.0 ** rng.integers(-3, 3, b[kind == 3].shape)
    return M.bf16(x)


@pytest.mark.parametrize("d,hkv", [(128, 1), (128, 3), (64, 2), (64, 5)])
@pytest.mark.parametrize("n", [1, 31, 64, 65, 200])
def test_put_keeps_the_nearest_numbers(d, hkv, n):
    rng = np.random.default_rng(d + hkv * 7 + n)
    k, v = wild(rng, (2, n, hkv, d)), wild(rng, (2, n, hkv, d))
    with pic.Store(pic.GQA, pic.FP4, hkv, d, d, 1024, n_layers=2) as store:
        store.put(5, n, dev(k, shift=n % 2), dev(v, shift=1), stream())
        assert store.usage() == ((n + 63) // 64 * 64, 1024, 1)
        for l in range(2):
            a, b = gather(store, [5, 5], 2 * n, hkv, d, layer=l)
            assert same(a, np.concatenate([M.stored(k[l])] * 2))
            assert same(b, np.concatenate([M.stored(v[l])] * 2))


def test_put_of_extremes():
    top = 3.3895313892515355e38                  # the largest bf16 number
    x = np.zeros((8, 1, 64))
    x[0, 0, :3] = [np.inf, 1e38, -np.inf]
    x[1, 0, :3] = [top, -top, 1e37]
    x[2, 0, :2] = [1.75 * 2.0 ** 126, 2.0 ** 120]
    x[3, 0, :4] = [2.0 ** -120, 2.0 ** -126, -2.0 ** -127, 2.0 ** -125]
    x[4, 0, :4] = [1.5 * 2.0 ** -126, 2.0 ** -126, 2.0 ** -130, -0.0]
    x[5, 0, :4] = [2.0 ** -127, 2.0 ** -128, 2.0 ** -133, -2.0 ** -127]
    x[6, 0, 33] = np.nan
    x[6, 0, 3] = 2.0
    x[7, 0, :2] = [np.nan, np.inf]
    x = M.bf16(x)
    with pic.Store(pic.GQA, pic.FP4, 1, 64, 64, 64) as store:
        store.put(1, 8, dev(x), dev(x[::-1].copy()), stream())
        a, b = gather(store, [1], 8, 1, 64)
        assert same(a, M.stored(x))
        assert same(b, M.stored(x[::-1]))


# name: d, hq, hkv, chunk lengths, links of each request, query tokens, own beyond the
# query (None: no own KV), sub-range starts, per-query limits, decode, pieces
FORMS = {
    "one_key": (128, 4, 2, (1,), [(0,)], (1,), None, False, False, True, 0),
    "one_key_64": (64, 2, 1, (1,), [(0,)], (1,), None, False, False, False, 0),
    "own_only": (128, 8, 2, (64,), [(), ()], (1, 3), (0, 70), False, False, True, 0),
    "nothing": (128, 4, 4, (64,), [(), (0,)], (2, 1), None, False, False, True, 0),
    "empty_request": (64, 4, 2, (64, 65), [(0,), (1, 0), ()], (0, 2, 0), (3, 0, 5), False, False, True, 0),
    "tails": (128, 8, 2, (63, 64, 65, 1, 130), [(0, 1, 2), (3, 4, 3), (2,)], (1, 2, 4), (31, 0, 64),
              False, False, True, 0),
    "tails_64": (64, 6, 3, (63, 64, 65, 1, 130), [(0, 1, 2), (3, 4, 3), (2,)], (1, 2, 8), (31, 0, 64),
                 False, False, True, 0),
    "pieces": (128, 32, 8, (200, 300, 64), [(0, 1), (1, 2, 0)], (1, 1), (40, 0), False, False, True, 5),
    "more_pieces_than_tiles": (64, 4, 1, (70, 64), [(0,), (1, 0)], (1, 2), (3, 90), False, False, True, 9),
    "prefill": (128, 8, 2, (150, 64, 70), [(0, 1), (2, 0), (1,)], (37, 5, 70), (4, 0, 100), False, False,
                False, 0),
    "prefill_64": (64, 6, 2, (150, 64, 70), [(0, 1), (2, 0), (1,)], (37, 130, 70), (4, 0, 100), False,
                   False, False, 0),
    "long_rows": (128, 4, 1, (300, 129), [(0, 1)], (200,), (9,), False, False, False, 0),
    "cross_only": (64, 8, 8, (100, 33), [(0, 1), (1,)], (65, 3), None, False, False, False, 0),
    "starts": (128, 8, 4, (65, 200, 129), [(0, 1, 2), (2, 2)], (20, 3), (0, 1), True, False, False, 0),
    "limits": (128, 8, 2, (65, 200, 129), [(0, 1, 2), (2, 2), (1,)], (20, 70, 9), None, False, True, False, 0),
    "limits_own": (64, 4, 2, (65, 200, 129), [(0, 1, 2), (2, 2), ()], (20, 70, 9), (0, 33, 1), True, True,
                   False, 0),
    "limits_decode": (128, 16, 2, (65, 200), [(0, 1), (1,)], (2, 1), None, False, True, True, 3),
    "group_of_nine": (128, 18, 2, (100, 90), [(0, 1), (1,)], (1, 2), (5, 0), False, False, True, 0),
    "group_of_forty": (64, 40, 1, (100, 90), [(0, 1), (1,)], (1, 2), (5, 0), False, False, True, 0),
    "many_links": (128, 4, 1, tuple(range(1, 70)), [tuple(range(69)), (5, 5, 5)], (3, 40), (0, 3), False,
                   False, False, 0),
}

# More work, with what can go wrong in long calls
MANY, MORE = (0,) * 14, (0,) * 28
BLOCKS = {
    "rows_80_and_6": (128, 16, 8, (1000, 65, 130), [MANY + (1, 2), (2,)], (40, 3), (5, 0), False, False, False, 0),
    "rows_2_blocks": (128, 16, 8, (1000, 1), [(1,) + MANY, (1,), ()], (150, 33, 2), (0, 64, 3), False, False,
                      False, 0),
    "rows_300_64": (64, 16, 8, (1000, 65, 130), [MORE + (1, 2), (1,)], (150, 3), (4, 100), False, False, False, 0),
    "long_own": (128, 8, 4, (700,), [(0,) * 38], (70,), (900,), False, False, False, 0),
    "long_own_64": (64, 8, 8, (700,), [(0,) * 38], (70,), (900,), False, False, False, 0),
    "starts_cross_only": (128, 16, 8, (1000, 65, 130), [MANY + (1, 2, 1), (1,)], (40, 60), None, True, False,
                          False, 0),
    "row_limits": (128, 16, 8, (1000, 65, 130), [MANY + (1, 2), (2,), (1, 0)], (140, 3, 40), None, False, True,
                   False, 0),
    "row_limits_64": (64, 16, 8, (1000, 65, 130), [MORE + (1, 2), (2,)], (140, 40), None, False, True, False, 0),
    "row_limits_own": (128, 16, 8, (1000, 65, 130), [MANY + (1, 2), (2,)], (70, 40), (0, 70), True, True, False, 0),
    "decode_pieces": (128, 64, 8, (1000, 65), [MANY + (1,), (1,)], (16, 9), (3, 0), False, False, True, 7),
    "odd_group": (64, 24, 8, (1000, 33), [MORE + (1,)], (45,), (20,), False, False, False, 0),
}
# Enough rows and work for the 256-row kernel (more than 128 rows, 12 tiles per CU or 24 of
# 64-wide heads; two of the forms above have them, too)
M25, M50 = (0,) * 26, (0,) * 50
WIDE = {
    "rows_160_and_6": (128, 16, 8, (1000, 65, 130), [M25 + (1, 2), (2,)], (80, 3), (5, 0), False, False, False, 0),
    "own_900": (128, 8, 4, (700,), [(0,) * 75], (70,), (900,), False, False, False, 0),
    "own_900_64": (64, 8, 8, (700,), [(0,) * 76], (140,), (900,), False, False, False, 0),
    "starts_blocks": (128, 16, 8, (1000, 65, 130), [M25 + (1, 2, 1), (1,)], (70, 60), None, True, False, False, 0),
    "row_limits_own_blocks": (128, 16, 8, (1000, 65, 130), [M25 + (1, 2), (2,)], (70, 40), (0, 70), True, True,
                              False, 0),
    "decode_blocks": (128, 128, 8, (1000, 65), [M25 + (1,), (1,)], (16, 9), (3, 0), False, False, True, 7),
    "row_limits_blocks": (128, 16, 8, (1000, 65, 130), [MANY + (1, 2), (2,), (1, 0)], (200, 3, 40), None, False, True,
                          False, 0),
    "row_limits_blocks_64": (64, 16, 8, (1000, 65, 130), [MORE + (1, 2), (2,)], (170, 40), None, False, True, False,
                             0),
    "odd_group_blocks": (64, 24, 8, (1000, 33), [M50 + (1,)], (45,), (20,), False, False, False, 0),
}
FORMS.update(BLOCKS)
FORMS.update(WIDE)
# Tables that just fit a kernel's arguments (one item and 110 links) and that do not
for n in (109, 110, 111):
    FORMS[f"links_{n}"] = (64, 4, 2, (3, 64, 65), [tuple(i % 3 for i in range(n))], (2,), None, False, False, True, 1)
ROWS_256 = ["rows_2_blocks", "rows_300_64"] + list(WIDE)


class Call:
    """A batch's inputs on the host and the GPU, and its reference."""

    def __init__(self, form, seed=0, shift=0, q_std=1.0):
        d, hq, hkv, lens, links, q_len, own, starts, limits, self.decode, self.pieces = FORMS[form]
        rng = np.random.default_rng(seed + sum(map(ord, form)))
        self.d, self.hq, self.hkv = d, hq, hkv
        draw = lambda *s: M.bf16(rng.standard_normal(s))  # noqa: E731
        self.raw = {i: (draw(n, hkv, d), draw(n, hkv, d)) for i, n in enumerate(lens)}
        self.links = links
        self.starts = [[64 if starts and lens[c] > 64 and j % 2 == 0 else 0 for j, c in enumerate(l)]
                       for l in links]
        off = lambda x: np.concatenate([[0], np.cumsum(x)]).astype(np.int32)  # noqa: E731
        self.q_off = off(q_len)
        self.own_off = None if own is None else off([a + b for a, b in zip(q_len, own)])
        self.q = M.bf16(q_std * rng.standard_normal((sum(q_len), hq, d)))
        ts = 0 if own is None else int(self.own_off[-1])
        self.k_own = None if own is None else draw(ts, hkv, d)
        self.v_own = None if own is None else draw(ts, hkv, d)
        doc = [sum(lens[c] - s for c, s in zip(l, st)) for l, st in zip(links, self.starts)]
        self.limits = None
        if limits:
            self.limits = np.concatenate([rng.integers(0, n + 1, m) for n, m in zip(doc, q_len)])
            self.limits[0] = 0
        self.scale = float(np.float32(1 / np.sqrt(d)))
        self.lens, self.shift = lens, shift

    def store(self, capacity=None):
        s = pic.Store(pic.GQA, pic.FP4, self.hkv, self.d, self.d,
                      capacity or sum((n + 63) // 64 * 64 for n in self.lens))
        for i, (k, v) in self.raw.items():
            s.put(i, k.shape[0], dev(k), dev(v), stream())
        return s

    def args(self):
        return ([0] + list(np.cumsum([len(l) for l in self.links])), [c for l in self.links for c in l],
                self.q_off, self.own_off)

    def kwargs(self):
        return dict(chunk_starts=[s for l in self.starts for s in l], q_doc_limits=self.limits)

    def tensors(self):
        own = (None, None) if self.k_own is None else (dev(self.k_own, self.shift), dev(self.v_own, self.shift))
        return (dev(self.q, self.shift),) + own

    def outputs(self):
        n = self.q.shape[0]
        out = torch.full((n * self.hq * self.d + self.shift,), 77, dtype=torch.int16, device="cuda")
        return (out[self.shift:].view(n, self.hq, self.d), torch.full((n, self.hq), 5.0, dtype=torch.float32,
                                                                   device="cuda"))

    def run(self, store, decode=None, pieces=None, entry=None, st=None):
        out, lse = self.outputs()
        decode = self.decode if decode is None else decode
        kw = self.kwargs()
        if decode:
            kw["num_splits"] = self.pieces if pieces is None else pieces
        f = entry or (pic.link_decode if decode else pic.link_attn)
        f(store, *self.args(), self.hq, *self.tensors(), self.scale, out, lse,
          stream=st or stream(), **kw)
        torch.cuda.synchronize()
        return host(out), lse.cpu().numpy().astype(np.float64)

    def reference(self):
        chunks = {i: (M.stored(k), M.stored(v)) for i, (k, v) in self.raw.items()}
        return M.batch(self.q, chunks, self.links, self.starts, self.k_own, self.v_own, self.q_off,
                       self.own_off, self.scale, self.limits)


def check(got, ref):
    (out, lse), (ro, rl, to, tl) = got, ref
    assert same(np.isfinite(lse), np.isfinite(rl)) and np.array_equal(lse[~np.isfinite(rl)], rl[~np.isfinite(rl)])
    f = np.isfinite(rl)
    bad = np.abs(lse[f] - rl[f]) - tl[f]
    assert (bad <= 0).all(), f"lse off its bound by {bad.max()}"
    over = np.abs(out - ro) - to
    assert not np.isnan(out).any() and (over <= 0).all(), f"out off its bound by {over.max()}"


@pytest.mark.parametrize("form", sorted(FORMS))
def test_link(form):
    c = Call(form)
    print(f"form {form}", flush=True)
    with c.store() as store:
        pic.prof_begin()
        got = c.run(store)
        name = pic.prof_end()[2]
        assert name == ("link_fp4_prefill_kernel" if form in ROWS_256 else "link_fp4_kernel")
        check(got, c.reference())


@pytest.mark.parametrize("form", ["tails", "prefill_64", "limits_own", "rows_80_and_6", "rows_300_64", "own_900"])
def test_unaligned_tensors(form):
    c = Call(form, seed=1, shift=3)
    with c.store() as store:
        check(c.run(store), c.reference())


@pytest.mark.parametrize("form", ["tails", "pieces", "tails_64"])
def test_decode_as_prefill_and_any_pieces(form):
    c = Call(form, seed=2)
    ref = c.reference()
    with c.store() as store:
        check(c.run(store, decode=False), ref)
        for s in (1, 2, 256):
            check(c.run(store, pieces=s), ref)


@pytest.mark.parametrize("std", [1e-3, 40.0])
def test_flat_and_sharp_softmax(std):
    for form in ("tails", "rows_80_and_6", "odd_group", "rows_160_and_6", "odd_group_blocks"):
        c = Call(form, seed=3, q_std=std)
        with c.store() as store:
            check(c.run(store), c.reference())


@pytest.mark.parametrize("form", ["tails", "pieces", "rows_80_and_6", "rows_300_64", "row_limits", "rows_160_and_6",
                                  "row_limits_blocks"])
@pytest.mark.parametrize("sign", [-1, 1])
def test_logits_far_from_zero(form, sign):
    """Every logit some hundreds below (above) zero: no probability may be formed against zero."""
    c = Call(form, seed=9)
    c.q = M.bf16(8 + 0.25 * c.q)
    c.raw = {i: (M.bf16(sign * 8 + k), v) for i, (k, v) in c.raw.items()}
    if c.k_own is not None:
        c.k_own = M.bf16(sign * 8 + c.k_own)
    with c.store() as store:
        check(c.run(store), c.reference())


@pytest.mark.parametrize("form", ["tails", "pieces", "limits_decode", "group_of_forty", "own_only", "decode_pieces",
                                  "decode_blocks"])
def test_noalloc_returns_the_same_bits(form):
    c = Call(form, seed=4)
    with c.store() as store:
        a, b = c.run(store), c.run(store, entry=pic.link_decode_noalloc)
        assert same(a[0], b[0]) and same(a[1], b[1])


@pytest.mark.parametrize("form", ["tails", "prefill", "limits", "pieces", "rows_2_blocks", "row_limits_64",
                                  "row_limits_blocks_64"])
def test_plans_and_captured_runs_return_the_same_bits(form):
    c = Call(form, seed=5)
    with c.store() as store:
        want = c.run(store)
        out, lse = c.outputs()
        t = c.tensors()
        plan = pic.LinkPlan(store, *c.args(), c.hq, mode=pic.DECODE if c.decode else pic.PREFILL,
                            num_splits=c.pieces if c.decode else 0, **c.kwargs())
        with plan:
            plan.run(0, *t, c.scale, out, lse, stream())
            torch.cuda.synchronize()
            assert same(host(out), want[0]) and same(lse.cpu().numpy().astype(np.float64), want[1])
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                plan.run(0, *t, c.scale, out, lse, stream())
            for k in range(3):
                out.fill_(k)
                lse.fill_(k)
                plan.run(0, *t, c.scale, *c.outputs(), stream())    # eager work in between
                g.replay()
                torch.cuda.synchronize()
                assert same(host(out), want[0]) and same(lse.cpu().numpy().astype(np.float64), want[1])


def test_calls_in_flight_on_two_streams():
    c, e = Call("rows_160_and_6", seed=6), Call("pieces", seed=6)
    with c.store() as s1, e.store() as s2:
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        outs = []
        for k in range(6):
            for x, s, st in ((c, s1, streams[0]), (e, s2, streams[1])):
                o, t = x.outputs(), x.tensors()
                torch.cuda.synchronize()
                kw = dict(x.kwargs(), **({"num_splits": x.pieces} if x.decode else {}))
                (pic.link_decode if x.decode else pic.link_attn)(
                    s, *x.args(), x.hq, *t, x.scale, *o, stream=st.cuda_stream, **kw)
                outs.append((x, o, t))
        torch.cuda.synchronize()
        refs = {id(c): c.reference(), id(e): e.reference()}
        for x, o, _ in outs:
            check((host(o[0]), o[1].cpu().numpy().astype(np.float64)), refs[id(x)])


@pytest.mark.parametrize("d", [64, 128])
def test_fragmented_chunks(d):
    """Chunks that removal has left in several runs of pages."""
    rng = np.random.default_rng(d)
    hkv = 2
    draw = lambda n: (M.bf16(rng.standard_normal((n, hkv, d))), M.bf16(rng.standard_normal((n, hkv, d))))  # noqa: E731
    with pic.Store(pic.GQA, pic.FP4, hkv, d, d, 6 * 64) as store:
        for i in range(6):
            k, v = draw(64)
            store.put(i, 64, dev(k), dev(v), stream())
        for i in (0, 2, 4):
            store.remove(i, stream())
        torch.cuda.synchronize()
        k, v = draw(170)
        store.put(9, 170, dev(k), dev(v), stream())
        a, b = gather(store, [9], 170, hkv, d)
        assert same(a, M.stored(k)) and same(b, M.stored(v))
        q = M.bf16(rng.standard_normal((3, 4, d)))
        out = torch.empty((3, 4, d), dtype=torch.int16, device="cuda")
        lse = torch.empty((3, 4), dtype=torch.float32, device="cuda")
        pic.link_attn(store, [0, 1], [9], [0, 3], None, 4, dev(q), None, None, 0.25, out, lse, stream=stream(),
                      chunk_starts=[64])
        torch.cuda.synchronize()
        ref = M.attend(q, M.stored(k)[64:], M.stored(v)[64:], 0.25, np.ones((3, 106), bool))
        check((host(out), lse.cpu().numpy().astype(np.float64)), ref)


@pytest.mark.parametrize("d,hkv,n_rows", [(64, 3, 5), (128, 2, 140), (128, 1, 900)])
def test_derived_rows(d, hkv, n_rows):
    """Single rows written into a derived chunk: their blocks change, nothing else does."""
    rng = np.random.default_rng(n_rows)
    n = 1000
    k, v = wild(rng, (2, n, hkv, d)), wild(rng, (2, n, hkv, d))
    rows = np.sort(rng.choice(n, n_rows, replace=False)).astype(np.int32)
    nk, nv = wild(rng, (n_rows, hkv, d)), wild(rng, (n_rows, hkv, d))
    with pic.Store(pic.GQA, pic.FP4, hkv, d, d, 4096, n_layers=2) as store:
        store.put(1, n, dev(k), dev(v), stream())
        store.derive(2, 1, rows, stream())
        store.write_rows(2, 1, rows, dev(nk), dev(nv), stream())
        want_k, want_v = M.stored(k), M.stored(v)
        for l in range(2):
            a, b = gather(store, [1], n, hkv, d, layer=l)
            assert same(a, want_k[l]) and same(b, want_v[l])
        want_k[1][rows], want_v[1][rows] = M.stored(nk), M.stored(nv)
        for l in range(2):
            a, b = gather(store, [2], n, hkv, d, layer=l)
            assert same(a, want_k[l]) and same(b, want_v[l])


def test_layers_past_32_bits_of_offset():
    """The last of 256 layers of a pool above 4 GiB."""
    rng = np.random.default_rng(0)
    layers, cap, hkv, d, n = 256, 16384, 8, 128, 70
    k, v = (M.bf16(rng.standard_normal((n, hkv, d))) for _ in range(2))
    kd = torch.zeros((layers, n, hkv, d), dtype=torch.int16, device="cuda")
    vd = torch.zeros_like(kd)
    kd[-1], vd[-1] = dev(k), dev(v)
    assert layers * cap * hkv * 2 * d * 17 // 32 > 1 << 32
    with pic.Store(pic.GQA, pic.FP4, hkv, d, d, cap, n_layers=layers) as store:
        store.put(3, n, kd, vd, stream())
        a, b = gather(store, [3], n, hkv, d, layer=layers - 1)
        assert same(a, M.stored(k)) and same(b, M.stored(v))
        q = M.bf16(rng.standard_normal((2, hkv, d)))
        out = torch.empty((2, hkv, d), dtype=torch.int16, device="cuda")
        lse = torch.empty((2, hkv), dtype=torch.float32, device="cuda")
        pic.link_decode(store, [0, 1], [3], [0, 2], None, hkv, dev(q), None, None, 0.1, out, lse,
                        stream=stream(), layer=layers - 1)
        torch.cuda.synchronize()
        ref = M.attend(q, M.stored(k), M.stored(v), float(np.float32(0.1)), np.ones((2, n), bool))
        check((host(out), lse.cpu().numpy().astype(np.float64)), ref)


def test_plan_of_every_layer():
    """A plan's run on each layer, own KV of the layer, over a chunk with rows written in one."""
    rng = np.random.default_rng(4)
    d, hkv, n, layers = 64, 2, 130, 3
    draw = lambda *s: M.bf16(rng.standard_normal(s))  # noqa: E731
    k, v = draw(layers, n, hkv, d), draw(layers, n, hkv, d)
    rows = np.array([0, 63, 64, 129], np.int32)
    nk, nv = draw(4, hkv, d), draw(4, hkv, d)
    q, ko, vo = draw(5, 6, d), draw(7, hkv, d), draw(7, hkv, d)
    with pic.Store(pic.GQA, pic.FP4, hkv, d, d, 1024, n_layers=layers) as store:
        store.put(1, n, dev(k), dev(v), stream())
        store.derive(2, 1, rows, stream())
        store.write_rows(2, 2, rows, dev(nk), dev(nv), stream())
        args = ([0, 2, 3], [2, 1, 2], [0, 2, 5], [0, 4, 7])
        with pic.LinkPlan(store, *args, 6, mode=pic.DECODE, chunk_starts=[64, 0, 128]) as plan:
            sk, sv = M.stored(k), M.stored(v)
            for l in range(layers):
                out = torch.empty((5, 6, d), dtype=torch.int16, device="cuda")
                lse = torch.empty((5, 6), dtype=torch.float32, device="cuda")
                plan.run(l, dev(q), dev(ko), dev(vo), 0.125, out, lse, stream())
                torch.cuda.synchronize()
                two = (sk[l].copy(), sv[l].copy())
                if l == 2:
                    two[0][rows], two[1][rows] = M.stored(nk), M.stored(nv)
                ref = M.batch(q, {1: (sk[l], sv[l]), 2: two}, [(2, 1), (2,)], [[64, 0], [128]], ko, vo,
                              args[2], args[3], 0.125)
                check((host(out), lse.cpu().numpy().astype(np.float64)), ref)


def test_pages_of_removed_chunks_are_taken_whole():
    """A short chunk on a page that held other rows: nothing of them is read."""
    rng = np.random.default_rng(5)
    d, hkv = 128, 1
    big = np.full((64, hkv, d), np.nan)
    k, v, q = (M.bf16(rng.standard_normal((3, hkv, d))) for _ in range(3))
    with pic.Store(pic.GQA, pic.FP4, hkv, d, d, 64) as store:
        store.put(1, 64, dev(big), dev(big), stream())
        store.remove(1, stream())
        store.put(2, 3, dev(k), dev(v), stream())
        out = torch.empty((3, hkv, d), dtype=torch.int16, device="cuda")
        lse = torch.empty((3, hkv), dtype=torch.float32, device="cuda")
        pic.link_attn(store, [0, 1], [2], [0, 3], None, hkv, dev(q), None, None, 0.125, out, lse, stream=stream())
        torch.cuda.synchronize()
        check((host(out), lse.cpu().numpy().astype(np.float64)),
              M.attend(q, M.stored(k), M.stored(v), 0.125, np.ones((3, 3), bool)))


def test_another_process_links_the_exported_store():
    import multiprocessing as mp

    import fp4_ipc_child
    rng = np.random.default_rng(6)
    d, hkv, n = 128, 2, 100
    k, v, q = (M.bf16(rng.standard_normal(s)) for s in ((n, hkv, d), (n, hkv, d), (4, 4, d)))
    with pic.Store(pic.GQA, pic.FP4, hkv, d, d, 256) as store:
        store.put(9, n, dev(k), dev(v), stream())
        blob = store.export()
        ctx = mp.get_context("spawn")
        results = ctx.Queue()
        child = ctx.Process(target=fp4_ipc_child.run, args=(blob, M.bits(q), results))
        child.start()
        try:
            got = results.get(timeout=100)
        finally:
            child.join(timeout=15)
        assert not isinstance(got, str), got
        out = got[0].view(np.uint16).astype(np.uint32) << 16
        check((out.view(np.float32).astype(np.float64), got[1].astype(np.float64)),
              M.attend(q, M.stored(k), M.stored(v), 0.125, np.ones((4, n), bool)))


def test_infinities_and_nan():
    """Infinite cached numbers are kept as the largest; a row that sees a NaN key is NaN,
    one whose limit hides it is not; a NaN query gives a NaN row and leaves the others."""
    rng = np.random.default_rng(8)
    d, n = 128, 100
    k, v = (M.bf16(rng.standard_normal((n, 1, d))) for _ in range(2))
    v[7, 0, 3] = np.inf
    k[90, 0, 5] = np.nan
    q = M.bf16(rng.standard_normal((3, 2, d)))
    q[2, 1, 9] = np.nan
    with pic.Store(pic.GQA, pic.FP4, 1, d, d, 128) as store:
        store.put(1, n, dev(k), dev(v), stream())
        out = torch.empty((3, 2, d), dtype=torch.int16, device="cuda")
        lse = torch.empty((3, 2), dtype=torch.float32, device="cuda")
        pic.link_attn(store, [0, 1], [1], [0, 3], None, 2, dev(q), None, None, 0.125, out, lse,
                      stream=stream(), q_doc_limits=[100, 90, 50])
        torch.cuda.synchronize()
        o, l = host(out), lse.cpu().numpy().astype(np.float64)
        assert np.isnan(o[0]).all() and np.isnan(l[0]).all()
        assert np.isnan(o[2, 1]).all() and np.isnan(l[2, 1])
        seen = np.arange(n)[None, :] < np.array([0, 90, 50])[:, None]
        keep = np.where(np.isnan(M.stored(k)), 0, M.stored(k))
        qq = np.where(np.isnan(q), 0, q)
        ref = M.attend(qq, keep, M.stored(v), 0.125, seen)
        rows = ([1, 1, 2], [0, 1, 0])
        check((o[rows], l[rows]), [x[rows] for x in ref])
