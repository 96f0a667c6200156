"""Calls over 4-bit stores as a server makes them: batches that fill the GPU uncut, calls of every
kind in flight on two streams over one store, and the read-back of many chunks. The reference and
its tolerances are those of test_gpu_fp4_values.py."""
import ctypes
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import fp4_model as M
from paper_2602_01519_amd import pic
from test_gpu_fp4 import dev, gather, host, same
from test_gpu_fp4_values import check

pytestmark = pytest.mark.gpu


def chunks(rng, lens, hkv, d):
    draw = lambda n: M.bf16(rng.standard_normal((n, hkv, d)))  # noqa: E731
    return {i: (draw(n), draw(n)) for i, n in enumerate(lens)}


def filled(raw, hkv, d):
    store = pic.Store(pic.GQA, pic.FP4, hkv, d, d, sum((len(k) + 63) // 64 * 64 for k, _ in raw.values()))
    for i, (k, v) in raw.items():
        store.put(i, len(k), dev(k), dev(v), torch.cuda.current_stream().cuda_stream)
    return store


def batch(rng, raw, hq, links, q_len, own=None, starts=None, limits=False, decode=False, pieces=0):
    """A batch over the chunks; own: own tokens beyond the query (None: no own KV)."""
    hkv, d = raw[0][0].shape[1:]
    off = lambda x: np.concatenate([[0], np.cumsum(x)]).astype(np.int32)  # noqa: E731
    c = SimpleNamespace(hq=hq, hkv=hkv, d=d, raw=raw, links=links, decode=decode, pieces=pieces,
                        scale=float(np.float32(d ** -0.5)))
    c.starts = [[0] * len(l) for l in links] if starts is None else starts
    c.q_off = off(q_len)
    draw = lambda n, h: M.bf16(rng.standard_normal((n, h, d)))  # noqa: E731
    c.q = draw(sum(q_len), hq)
    c.own_off = c.k_own = c.v_own = c.limits = None
    if own is not None:
        c.own_off = off([a + b for a, b in zip(q_len, own)])
        c.k_own, c.v_own = draw(c.own_off[-1], hkv), draw(c.own_off[-1], hkv)
    if limits:
        doc = [sum(len(raw[i][0]) - s for i, s in zip(l, st)) for l, st in zip(links, c.starts)]
        c.limits = np.concatenate([rng.integers(0, n + 1, m) for n, m in zip(doc, q_len)]).astype(np.int32)
    c.t = (dev(c.q), None if own is None else dev(c.k_own), None if own is None else dev(c.v_own))
    c.args = (off([len(l) for l in links]), [i for l in links for i in l], c.q_off, c.own_off)
    c.kw = dict(chunk_starts=[s for l in c.starts for s in l], q_doc_limits=c.limits)
    return c


def buffers(c):
    return (torch.full(c.q.shape, 77, dtype=torch.int16, device="cuda"),
            torch.full(c.q.shape[:2], 5.0, dtype=torch.float32, device="cuda"))


def enqueue(c, store, out, lse, stream):
    kw = dict(c.kw, num_splits=c.pieces) if c.decode else c.kw
    (pic.link_decode if c.decode else pic.link_attn)(store, *c.args, c.hq, *c.t, c.scale, out, lse, stream=stream, **kw)


def result(out, lse):
    return host(out), lse.cpu().numpy().astype(np.float64)


def graph_nodes(graph):
    n = ctypes.c_size_t()
    f = pic.lib().hipGraphGetNodes
    f.argtypes, f.restype = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p], ctypes.c_int
    assert f(graph.raw_cuda_graph(), None, ctypes.byref(n)) == 0
    return n.value


# head width, query heads of 8 kv heads, query tokens, own tokens beyond them, starts
UNCUT = {
    # 8 requests of 4 row blocks x 8 heads: one round of the 256 CUs, tables as an argument
    "even": (128, 32, (256,) * 8, 0, False),
    # 16 of them: one round of two workgroups per CU
    "even_64": (64, 32, (256,) * 16, 33, False),
    # more than two rounds, row blocks of a unit side by side, the order of the requests
    # searched, tables copied (24 requests: 1536 B of items, 3840 of links)
    "ragged": (128, 32, tuple(256 - 13 * i % 101 for i in range(24)), 5, False),
    "ragged_64": (64, 32, tuple(256 - 11 * i % 83 for i in range(40)), 0, True),
    "group_of_three": (128, 24, tuple(342 - 17 * i % 90 for i in range(24)), None, True),
}


@pytest.mark.parametrize("form", sorted(UNCUT))
def test_batches_that_are_not_cut(form):
    """The 256-row kernel writing its outputs itself: one kernel in a plan's run, no combine."""
    d, hq, q_len, extra, starts = UNCUT[form]
    rng = np.random.default_rng(len(q_len))
    raw = chunks(rng, (512, 130, 300, 65), 8, d)
    links = [(0, 1, 2) if i % 3 else (2, 3, 0, 1) for i in range(len(q_len))]
    if extra == 0 and d == 128:
        links = [(0, 1, 2)] * len(q_len)
    c = batch(rng, raw, hq, links, q_len, None if extra is None else [extra] * len(q_len),
              [[64 if j == 0 else 0 for j in range(len(l))] for l in links] if starts else None)
    st = torch.cuda.current_stream().cuda_stream
    with filled(raw, 8, d) as store:
        out, lse = buffers(c)
        pic.prof_begin()
        enqueue(c, store, out, lse, st)
        assert pic.prof_end()[2] == "link_fp4_prefill_kernel"
        torch.cuda.synchronize()
        got = result(out, lse)
        check(c, got)
        with pic.LinkPlan(store, *c.args, c.hq, **c.kw) as plan:
            a, b = buffers(c)
            plan.run(0, *c.t, c.scale, a, b, st)
            torch.cuda.synchronize()
            assert all(same(x, y) for x, y in zip(got, result(a, b)))
            g = torch.cuda.CUDAGraph(keep_graph=True)
            with torch.cuda.graph(g):
                plan.run(0, *c.t, c.scale, a, b, torch.cuda.current_stream().cuda_stream)
            assert graph_nodes(g) == 1


@pytest.mark.parametrize("d", [64, 128])
def test_calls_of_every_kind_in_flight_over_one_store(d):
    """32 calls on two streams, back to back: they pass through the store's staging slots four
    times, with tables copied and as an argument, in pieces and not, with both kernels."""
    rng = np.random.default_rng(d)
    raw = chunks(rng, (512, 130, 300, 65, 700, 64), 8, d)
    kinds = [
        lambda: batch(rng, raw, 32, [(0, 1, 2)] * 8, (256,) * 8, [0] * 8),
        lambda: batch(rng, raw, 16, [(4, 0, 3, 2, 1)], (37,), [20]),
        lambda: batch(rng, raw, 32, [(4, 0, 3), (1, 2), (4, 4, 5, 0)] * 7, (1, 4, 2) * 7, [9] * 21, decode=True, pieces=3),
        lambda: batch(rng, raw, 32, [(4, 0, 3, 1), (2, 4)] * 3, (200, 61) * 3, limits=True),
    ]
    calls = [kinds[i % 4]() for i in range(16)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    with filled(raw, 8, d) as store:
        outs = [[buffers(c), buffers(c)] for c in calls]
        torch.cuda.synchronize()
        for k in range(2):
            for i, c in enumerate(calls):
                enqueue(c, store, *outs[i][k], streams[(i + i // 4 + k) % 2].cuda_stream)
        torch.cuda.synchronize()
        for c, (a, b) in zip(calls, outs):
            first = result(*a)
            assert all(same(x, y) for x, y in zip(first, result(*b)))
            check(c, first)


@pytest.mark.parametrize("d,hkv", [(64, 3), (128, 2)])
def test_read_back_of_many_chunks(d, hkv):
    """150 ids, more than one launch lists, one of them a chunk in several runs of pages."""
    rng = np.random.default_rng(d)
    raw = chunks(rng, (1, 63, 64, 65, 130, 7), hkv, d)
    more = chunks(rng, (300,), hkv, d)[0]
    st = torch.cuda.current_stream().cuda_stream
    with pic.Store(pic.GQA, pic.FP4, hkv, d, d, 20 * 64) as store:
        for i in range(100, 104):          # every second page is freed again
            store.put(i, 64, dev(raw[2][0]), dev(raw[2][1]), st)
            store.put(200 + i, 64, dev(raw[2][0]), dev(raw[2][1]), st)
        for i, (k, v) in raw.items():
            store.put(i, len(k), dev(k), dev(v), st)
        for i in range(100, 104):
            store.remove(i, st)
        torch.cuda.synchronize()
        store.put(9, 300, dev(more[0]), dev(more[1]), st)
        raw[9] = more
        ids = [int(x) for x in rng.choice(sorted(raw), 150)]
        assert 9 in ids
        n = sum(len(raw[i][0]) for i in ids)
        a, b = gather(store, ids, n + 1, hkv, d)
        assert same(a[:n], np.concatenate([M.stored(raw[i][0]) for i in ids]))
        assert same(b[:n], np.concatenate([M.stored(raw[i][1]) for i in ids]))
        untouched = host(torch.full((hkv, d), 77, dtype=torch.int16))
        assert same(a[n], untouched) and same(b[n], untouched)
