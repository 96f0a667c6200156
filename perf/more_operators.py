"""Growing chunks, link attention of requests that share their documents, and link attention
over selected blocks, as cases for performance measurement.

  append  new tokens of a batch are rotated and appended to the requests' chunks
          (Store.append), the chunks read back, and the tokens taken back
  shared  link attention of requests of which groups link the same documents
          (link_shared, or a plan of it)
  sparse  link attention over the blocks of 64 linked tokens that score best
          (link_sparse over a BlockIndex)

`run` computes the plain form (elementary torch operations) unless `own` is set; then it
makes the calls of paper_2602_01519_amd.pic. A case is a dict of plain values; its ragged
sizes come from its "shape" number, tensor values from the seed.

Blocks: every linked chunk is cut into blocks of 64 tokens (its last one may be shorter). A
block's summary is the mean of its keys, rounded to bf16, for each kv head; a query token's
score of a block, for each kv head, is the largest product of the summary with a query head
of that group. A query token takes the first `first` and the last `last` blocks of its request
and the best scored others, `blocks` in all; equal scores go to the lower block.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False


def _named(name, c):
    return c if name is None else {"name": name, **c}


def _append(name=None, *, dk, dv, hkv, hq, batch, have_lo, have_hi, add_lo, add_hi, rot_at, rot,
            dtype="bf16", kind="gqa", layout="half", scaling="none", theta=10000.0, factor=1.0,
            far=4096, fused=True, shape=1):
    return _named(name, dict(flow="append", dk=dk, dv=dv, hkv=hkv, hq=hq, batch=batch,
                             have_lo=have_lo, have_hi=have_hi, add_lo=add_lo, add_hi=add_hi,
                             rot_at=rot_at, rot=rot, dtype=dtype, kind=kind, layout=layout,
                             scaling=scaling, theta=theta, factor=factor, far=far, fused=fused,
                             shape=shape))


def _shared(name=None, *, hq, hkv, d, groups, per_lo, per_hi, links_lo, links_hi, len_lo, len_hi,
            mine_lo=0, mine_hi=0, q_lo=1, q_hi=1, own_lo=0, own_hi=0, dtype="bf16", plan=False, shape=1):
    return _named(name, dict(flow="shared", hq=hq, hkv=hkv, d=d, groups=groups, per_lo=per_lo,
                             per_hi=per_hi, links_lo=links_lo, links_hi=links_hi, len_lo=len_lo,
                             len_hi=len_hi, mine_lo=mine_lo, mine_hi=mine_hi, q_lo=q_lo, q_hi=q_hi,
                             own_lo=own_lo, own_hi=own_hi, dtype=dtype, plan=plan, shape=shape))


def _sparse(name=None, *, hq, hkv, d, batch, links_lo, links_hi, len_lo, len_hi, blocks, first=1,
            last=1, q_lo=1, q_hi=1, own_lo=1, own_hi=1, dtype="bf16", shape=1):
    return _named(name, dict(flow="sparse", hq=hq, hkv=hkv, d=d, batch=batch, links_lo=links_lo,
                             links_hi=links_hi, len_lo=len_lo, len_hi=len_hi, blocks=blocks,
                             first=first, last=last, q_lo=q_lo, q_hi=q_hi, own_lo=own_lo,
                             own_hi=own_hi, dtype=dtype, shape=shape))


def listed():
    return [
        # One generated token for each request of a full batch: launches.
        _append("append_step", dk=128, dv=128, hkv=8, hq=32, batch=64, have_lo=20, have_hi=200,
                add_lo=1, add_hi=1, rot_at=0, rot=128, theta=500000.0, scaling="banded", factor=8.0,
                far=130000),
        # Questions of a prefill batch enter their requests' caches.
        _append("append_prefill", dk=128, dv=128, hkv=8, hq=32, batch=16, have_lo=0, have_hi=0,
                add_lo=512, add_hi=512, rot_at=0, rot=128, theta=500000.0, scaling="banded",
                factor=8.0, far=130000, shape=2),
        # Latent rows of MLA, the rotated part at their end; ragged continuations.
        _append("append_latent", kind="mla", dk=576, dv=512, hkv=1, hq=16, batch=24, have_lo=1,
                have_hi=300, add_lo=3, add_hi=150, rot_at=512, rot=64, layout="interleaved",
                scaling="yarn", factor=40.0, far=160000, fused=False, shape=3),
        # Eight users ask about the same few documents, one decode step: latency.
        _shared("shared_few", hq=32, hkv=8, d=128, groups=1, per_lo=8, per_hi=8, links_lo=6,
                links_hi=6, len_lo=200, len_hi=900, own_lo=20, own_hi=90, plan=True, shape=4),
        # One decode step of a batch whose 64 requests link the same 16 documents.
        _shared("shared_step", hq=32, hkv=8, d=128, groups=1, per_lo=64, per_hi=64, links_lo=16,
                links_hi=16, len_lo=1024, len_hi=1024, own_lo=1, own_hi=255, plan=True, shape=5),
        # Ragged groups over long document sets: the largest.
        _shared("shared_long", hq=32, hkv=8, d=128, groups=4, per_lo=30, per_hi=60, links_lo=40,
                links_hi=64, len_lo=700, len_hi=1024, mine_lo=0, mine_hi=2, own_lo=1, own_hi=300,
                plan=True, shape=6),
        # Questions of a few dozen tokens about common documents, 64-wide heads.
        _shared("shared_questions", hq=24, hkv=6, d=64, groups=3, per_lo=3, per_hi=9, links_lo=3,
                links_hi=9, len_lo=90, len_hi=1000, mine_lo=0, mine_hi=3, q_lo=5, q_hi=60, own_lo=0,
                own_hi=100, shape=7),
        # One user's decode step over a dozen documents: latency.
        _sparse("sparse_one", hq=32, hkv=8, d=128, batch=1, links_lo=12, links_hi=12, len_lo=300,
                len_hi=1000, blocks=24, own_lo=40, own_hi=40, shape=8),
        # One decode step of a batch over 16 documents each, an eighth of the blocks.
        _sparse("sparse_step", hq=32, hkv=8, d=128, batch=32, links_lo=16, links_hi=16, len_lo=1024,
                len_hi=1024, blocks=32, own_lo=1, own_hi=255, shape=9),
        # Long document sets, few requests.
        _sparse("sparse_long", hq=32, hkv=8, d=128, batch=12, links_lo=40, links_hi=64, len_lo=700,
                len_hi=1024, blocks=64, first=2, last=4, own_lo=1, own_hi=300, shape=10),
        # fp32 with few 64-wide heads, some tokens checked at once.
        _sparse("sparse_tokens", hq=8, hkv=2, d=64, batch=9, links_lo=2, links_hi=14, len_lo=60,
                len_hi=700, blocks=12, first=0, last=2, q_lo=1, q_hi=4, own_lo=4, own_hi=50,
                dtype="f32", shape=11),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _span(rng, lo, hi):
    return sorted((_log_int(rng, lo, hi), _log_int(rng, lo, hi)))


def draw(rng):
    """One more case of the listed ranges, no more work than the largest of its flow."""
    flow = rng.choice(["append", "shared", "sparse"])
    most = {}
    for c in listed():
        w = work(c)
        for k in w:
            most[c["flow"], k] = max(w[k], most.get((c["flow"], k), 0.0))
    while True:
        hkv = rng.choice([1, 2, 3, 4, 6, 8])
        hq = hkv * rng.choice([1, 2, 3, 4, 5, 8])
        d = rng.choice([64, 128, 128])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        shape = rng.randrange(1 << 20)
        if flow == "append":
            rot = 2 * rng.randint(4, 64)
            rest = 8 * rng.randint(0, 8) + -rot % 8
            mla = rng.random() < 0.3
            have_lo, have_hi = _span(rng, 1, 300)
            add_lo, add_hi = rng.choice([(1, 1), _span(rng, 1, 6), _span(rng, 1, 600)])
            c = _append(kind="mla" if mla else "gqa", dk=rot + rest, dv=rot + rest if not mla else 8 * rng.randint(1, (rot + rest) // 8),
                        hkv=1 if mla else hkv, hq=hq, batch=_log_int(rng, 1, 64),
                        have_lo=have_lo - 1, have_hi=have_hi, add_lo=add_lo, add_hi=add_hi,
                        rot_at=rng.choice([0, rest]), rot=rot, dtype=dtype,
                        layout=rng.choice(["half", "interleaved"]),
                        scaling=rng.choice(["none", "linear", "banded", "yarn"]),
                        theta=rng.choice([10000.0, 500000.0]), factor=float(rng.choice([2, 8, 40])),
                        far=_log_int(rng, 16, 1000000), fused=rng.random() < 0.6, shape=shape)
        else:
            links_lo, links_hi = _span(rng, 1, 64)
            len_lo, len_hi = _span(rng, 1, 1100)
            own_lo, own_hi = _span(rng, 1, 300)
            if flow == "shared":
                q_lo, q_hi = rng.choice([(1, 1), (1, 1), _span(rng, 1, 6), _span(rng, 1, 60)])
                per_lo, per_hi = _span(rng, 1, 64)
                mine_lo, mine_hi = rng.choice([(0, 0), (0, 2), (1, 4)])
                own_kv = rng.random() < 0.8
                c = _shared(hq=hq, hkv=hkv, d=d, groups=rng.randint(1, 6), per_lo=per_lo, per_hi=per_hi,
                            links_lo=links_lo, links_hi=links_hi, len_lo=len_lo, len_hi=len_hi,
                            mine_lo=mine_lo, mine_hi=mine_hi, q_lo=q_lo, q_hi=q_hi,
                            own_lo=own_lo if own_kv else 0, own_hi=own_hi if own_kv else 0, dtype=dtype,
                            plan=rng.random() < 0.6, shape=shape)
            else:
                q_lo, q_hi = rng.choice([(1, 1), (1, 1), _span(rng, 1, 6)])
                blocks = _log_int(rng, 4, 96)
                c = _sparse(hq=hq, hkv=hkv, d=d, batch=_log_int(rng, 1, 48), links_lo=links_lo,
                            links_hi=links_hi, len_lo=len_lo, len_hi=len_hi, blocks=blocks,
                            first=rng.randint(0, 2), last=rng.randint(0, 2), q_lo=q_lo, q_hi=q_hi,
                            own_lo=own_lo, own_hi=own_hi, dtype=dtype, shape=shape)
        w = work(c)
        if all(w[k] <= most[flow, k] for k in w):
            return c


# ---------------------------------------------------------------------------
# Shapes of a case

class _Shape:
    """Token counts, links and groups of a case."""

    def __init__(self, c):
        r = random.Random(c["shape"])
        span = lambda k: r.randint(c[k + "_lo"], c[k + "_hi"])  # noqa: E731
        if c["flow"] == "append":
            self.have = [span("have") for _ in range(c["batch"])]
            self.add = [span("add") for _ in range(c["batch"])]
            return
        self.lens = []                     # tokens of every chunk

        def links(n):
            at = len(self.lens)
            self.lens += [span("len") for _ in range(n)]
            return list(range(at, at + n))

        if c["flow"] == "shared":
            self.per = [span("per") for _ in range(c["groups"])]
            self.common = [links(span("links")) for _ in self.per]
            self.batch = sum(self.per)
            self.mine = [links(span("mine")) for _ in range(self.batch)]
        else:
            self.batch = c["batch"]
            self.mine = [links(span("links")) for _ in range(self.batch)]
        self.q = [span("q") for _ in range(self.batch)]
        self.own_kv = c["own_hi"] > 0
        self.own = [max(n, span("own")) if self.own_kv else 0 for n in self.q]
        self.at = np.concatenate([[0], np.cumsum(self.lens)]).astype(np.int64)

    def rows(self, ids):
        """Cache rows of the chunks `ids`, in order."""
        return np.concatenate([np.arange(self.at[i], self.at[i + 1]) for i in ids] + [np.zeros(0, np.int64)])


def _offsets(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def _chunk_id(i):
    return 0x5851F42D4C957F2D * (i + 1) & 0x7FFFFFFFFFFFFFFF


def _width(c):
    return 4 if c["dtype"] == "f32" else 2


def work(case):
    """Bytes and operations of one pass: inputs read once, outputs written once, only the
    pairs that see each other. sparse: the summaries, and the blocks that each query token
    and kv head takes (once where they are all of the request's)."""
    c, s, es = case, _Shape(case), _width(case)
    if c["flow"] == "append":
        row = c["hkv"] * (c["dk"] + (c["dv"] if c["kind"] == "gqa" else 0))
        new, q = sum(s.add) * row, sum(s.add) * c["hq"] * c["dk"]
        # tokens in, their rows and the queries out; the chunks read back
        return {"bytes": es * (2.0 * (new + q) + 2.0 * (new + sum(s.have) * row)) + 4.0 * sum(s.add),
                "flops": 3.0 * sum(s.add) * (c["hkv"] + c["hq"]) * c["rot"]}
    row, tq = c["hkv"] * 2 * c["d"] * es, sum(s.q)
    io = sum(s.own) * row + tq * c["hq"] * (2 * c["d"] * es + 4)
    pair = c["hq"] * 4 * c["d"]
    pairs = sum(i + 1 + n - m for m, n in zip(s.q, s.own) for i in range(m) if n)
    count = lambda ids: sum(s.lens[i] for i in ids)  # noqa: E731
    if c["flow"] == "shared":
        at = 0
        for per, common in zip(s.per, s.common):
            pairs += sum(s.q[at:at + per]) * count(common)
            at += per
        pairs += sum(m * count(l) for m, l in zip(s.q, s.mine))
        return {"bytes": float(io + sum(s.lens) * row), "flops": float(pairs * pair)}
    bytes_, flops = io, 0
    for m, l in zip(s.q, s.mine):
        n = sum((s.lens[i] + 63) // 64 for i in l)
        take = min(n, c["blocks"])
        tokens = min(take * 64, count(l))
        bytes_ += n * c["hkv"] * c["d"] * 2 + min(m * tokens, count(l)) * row + m * c["hkv"] * c["blocks"] * 4
        flops += m * n * c["hq"] * 2 * c["d"] + m * tokens * pair
    return {"bytes": float(bytes_), "flops": float(flops + pairs * pair)}


# ---------------------------------------------------------------------------
# Inputs

class _Draw:
    """Seeded N(0, 1) tensors, one after another."""

    def __init__(self, c, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed * 1000003 + c["shape"])
        self.dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16

    def __call__(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda", dtype=torch.float32).to(self.dtype)


class _State:
    pass


_LENGTH, _LOW, _HIGH, _FAST, _SLOW = 4096, 1.0, 4.0, 32.0, 1.0


def _frequencies(c):
    """Angle per position of every rotated pair, in 64 bits, and the factor of cos and sin."""
    half = c["rot"] // 2
    f = c["theta"] ** (-np.arange(half, dtype=np.float64) / half)
    if c["scaling"] == "linear":
        return f / c["factor"], 1.0
    if c["scaling"] == "banded":
        keep = np.clip((_LENGTH * f / (2 * np.pi) - _LOW) / (_HIGH - _LOW), 0.0, 1.0)
        return f * (keep + (1.0 - keep) / c["factor"]), 1.0
    if c["scaling"] == "yarn":
        at = lambda turns: half * math.log(_LENGTH / (turns * 2 * math.pi)) / math.log(c["theta"])  # noqa: E731
        lo = max(math.floor(at(_FAST)), 0)
        hi = min(math.ceil(at(_SLOW)), c["rot"] - 1)
        ramp = np.clip((np.arange(half) - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return f * ((1.0 - ramp) + ramp / c["factor"]), 0.1 * math.log(c["factor"]) + 1.0
    return f, 1.0


def _append_inputs(c, s, rnd):
    """Cached tokens of every chunk, the new ones (k, v, q: slices of one projection's rows
    where fused), and their positions."""
    gqa, n, m = c["kind"] == "gqa", sum(s.add), sum(s.have)
    k_have = rnd(m, c["hkv"], c["dk"])
    v_have = rnd(m, c["hkv"], c["dv"]) if gqa else None
    if c["fused"]:
        wq, wk, wv = c["hq"] * c["dk"], c["hkv"] * c["dk"], c["hkv"] * c["dv"] if gqa else 0
        x = rnd(n, wq + wk + wv)
        q, k = x[:, :wq].view(n, c["hq"], c["dk"]), x[:, wq:wq + wk].view(n, c["hkv"], c["dk"])
        v = x[:, wq + wk:].view(n, c["hkv"], c["dv"]) if gqa else None
    else:
        q, k = rnd(n, c["hq"], c["dk"]), rnd(n, c["hkv"], c["dk"])
        v = rnd(n, c["hkv"], c["dv"]) if gqa else None
    first = torch.randint(0, c["far"], (c["batch"],), generator=rnd.gen, device="cuda", dtype=torch.int32)
    add = torch.tensor(s.add, device="cuda")
    pos = torch.repeat_interleave(first, add) + torch.cat([torch.arange(a, device="cuda", dtype=torch.int32) for a in s.add])
    return k_have, v_have, k, v, q, pos.to(torch.int32)


def _link_inputs(c, s, rnd):
    """K and V of all chunks, queries, own K and V."""
    n, tq, ts = sum(s.lens), sum(s.q), sum(s.own)
    k, v = rnd(n, c["hkv"], c["d"]), rnd(n, c["hkv"], c["d"])
    q = rnd(tq, c["hq"], c["d"])
    if not s.own_kv:
        return k, v, q, None, None
    return k, v, q, rnd(ts, c["hkv"], c["d"]), rnd(ts, c["hkv"], c["d"])


def _stream():
    return torch.cuda.current_stream().cuda_stream


def prepare(case, seed):
    c = case
    st = _State()
    st.c, st.s = c, _Shape(c)
    rnd = _Draw(c, seed)
    if c["flow"] == "append":
        _prepare_append(st, rnd)
        return st
    s = st.s
    k, v, st.q, st.k_own, st.v_own = _link_inputs(c, s, rnd)
    st.scale = float(np.float32(1.0 / math.sqrt(c["d"])))
    st.q_at, st.own_at = _offsets(s.q), _offsets(s.own)
    if own:
        from paper_2602_01519_amd import pic
        st.out = torch.empty_like(st.q)
        st.lse = torch.empty(st.q.shape[:2], dtype=torch.float32, device="cuda")
        st.store = pic.Store(pic.GQA, pic.F32 if c["dtype"] == "f32" else pic.BF16, c["hkv"], c["d"],
                             c["d"], sum((n + 63) // 64 * 64 for n in s.lens))
        for i, n in enumerate(s.lens):
            st.store.put(_chunk_id(i), n, k[s.at[i]:s.at[i + 1]], v[s.at[i]:s.at[i + 1]], _stream())
        ids = lambda lists: np.array([_chunk_id(i) for l in lists for i in l], dtype=np.uint64)  # noqa: E731
        st.offsets, st.ids = _offsets([len(l) for l in s.mine]), ids(s.mine)
        st.own_offsets = st.own_at if s.own_kv else None
        if c["flow"] == "shared":
            st.groups = (_offsets(s.per), _offsets([len(l) for l in s.common]), ids(s.common))
            if c["plan"]:
                st.plan = pic.SharedLinkPlan(st.store, *st.groups, st.offsets, st.ids, st.q_at,
                                             st.own_offsets, c["hq"])
        else:
            st.index = pic.BlockIndex(st.store)
            st.index.update(ids([range(len(s.lens))]), stream=_stream())
            st.taken = torch.empty(len(st.q), c["hkv"], c["blocks"], dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()        # k and v are freed here
        return st
    st.k, st.v = k, v
    on = lambda ids: torch.from_numpy(s.rows(ids)).cuda()  # noqa: E731
    st.mine = [on(l) for l in s.mine]
    if c["flow"] == "shared":
        st.common = [on(l) for l in s.common]
        return st
    # the summaries, as a program keeps them beside the cache, and every linked row's block
    st.means, st.block = [], []
    for l, rows in zip(s.mine, st.mine):
        n, block = _blocks(s, l)
        st.block.append(block)
        total = torch.zeros(n, c["hkv"], c["d"], dtype=torch.float64, device="cuda")
        total.index_add_(0, block, k[rows].double())
        size = torch.bincount(block, minlength=n).double()
        st.means.append((total / size[:, None, None]).float().to(torch.bfloat16))
    return st


def _blocks(s, links):
    """Blocks of a request's links and the block of each of their rows."""
    of, at = [], 0
    for i in links:
        of.append(torch.arange(s.lens[i], device="cuda") // 64 + at)
        at += (s.lens[i] + 63) // 64
    return at, torch.cat(of)


def _prepare_append(st, rnd):
    c, s = st.c, st.s
    k_have, v_have, st.k, st.v, st.q, st.pos = _append_inputs(c, s, rnd)
    total = sum(s.have) + sum(s.add)
    f, st.mag = _frequencies(c)
    st.freq = torch.from_numpy(f).cuda()
    st.q_out = torch.empty(st.q.shape, dtype=st.q.dtype, device="cuda")
    st.kc = torch.empty(total, c["hkv"], c["dk"], dtype=st.q.dtype, device="cuda")
    st.vc = None if st.v is None else torch.empty(total, c["hkv"], c["dv"], dtype=st.q.dtype, device="cuda")
    at_have = _offsets(s.have)
    if own:
        from paper_2602_01519_amd import pic
        dt = pic.F32 if c["dtype"] == "f32" else pic.BF16
        room = sum((h + a + 63) // 64 * 64 for h, a in zip(s.have, s.add))
        st.store = pic.Store(pic.GQA if c["kind"] == "gqa" else pic.MLA, dt, c["hkv"], c["dk"], c["dv"], room)
        st.ids = np.array([_chunk_id(i) for i in range(c["batch"])], dtype=np.uint64)
        for i in range(c["batch"]):
            st.store.open(st.ids[i], s.have[i] + s.add[i])
        st.store.append(st.ids, at_have, k_have, v_have, stream=_stream())
        st.offsets, st.have = _offsets(s.add), np.array(s.have, dtype=np.int64)
        st.rope = pic.Rope(dt, pic.ROPE_HALF if c["layout"] == "half" else pic.ROPE_INTERLEAVED,
                           c["dk"], c["rot_at"], c["rot"], theta=c["theta"],
                           scaling={"none": pic.ROPE_PLAIN, "linear": pic.ROPE_LINEAR,
                                    "banded": pic.ROPE_BANDED, "yarn": pic.ROPE_YARN}[c["scaling"]],
                           factor=c["factor"], original_len=_LENGTH, band_low=_LOW, band_high=_HIGH,
                           turns_fast=_FAST, turns_slow=_SLOW, magnitude=st.mag)
        torch.cuda.synchronize()
        return
    # a cache of whole sequences: the cached tokens in place, the rows of the new ones
    ends = _offsets([h + a for h, a in zip(s.have, s.add)])
    st.rows = torch.cat([torch.arange(e - a, e) for e, a in zip(ends[1:].tolist(), s.add)]).cuda()
    kept = torch.cat([torch.arange(e, e + h) for e, h in zip(ends[:-1].tolist(), s.have)]).cuda()
    st.kc[kept] = k_have
    if st.vc is not None:
        st.vc[kept] = v_have


# ---------------------------------------------------------------------------
# One pass

def run(st):
    if own:
        return _run_own(st)
    if st.c["flow"] == "append":
        return _appended(st)
    return _shared_form(st) if st.c["flow"] == "shared" else _sparse_form(st)


def _run_own(st):
    from paper_2602_01519_amd import pic
    c, stream = st.c, _stream()
    if c["flow"] == "append":
        st.store.append(st.ids, st.offsets, st.k, st.v, rope=st.rope, positions=st.pos, q=st.q,
                        q_out=st.q_out, stream=stream)
        pic.debug_gather(st.store, st.ids, st.kc, st.vc, stream)
        st.store.truncate(st.ids, st.have, stream)
        return [st.q_out, st.kc] + ([] if st.vc is None else [st.vc])
    if c["flow"] == "sparse":
        pic.link_sparse(st.index, st.offsets, st.ids, st.q_at, st.own_offsets, c["hq"], c["blocks"],
                        st.q, st.k_own, st.v_own, st.scale, st.out, st.lse, keep_first=c["first"],
                        keep_last=c["last"], blocks=st.taken, stream=stream)
        return [st.out, st.lse, st.taken]
    if c["plan"]:
        st.plan.run(0, st.q, st.k_own, st.v_own, st.scale, st.out, st.lse, stream)
    else:
        pic.link_shared(st.store, *st.groups, st.offsets, st.ids, st.q_at, st.own_offsets, c["hq"],
                        st.q, st.k_own, st.v_own, st.scale, st.out, st.lse, stream=stream)
    return [st.out, st.lse]


# ---------------------------------------------------------------------------
# The plain forms

def _turned(c, x, cos, sin):
    x = x.float()
    a, r = c["rot_at"], c["rot"]
    y = x.clone()
    if c["layout"] == "half":
        lo, hi = slice(a, a + r // 2), slice(a + r // 2, a + r)
    else:
        lo, hi = slice(a, a + r, 2), slice(a + 1, a + r, 2)
    y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
    y[..., hi] = x[..., lo] * sin + x[..., hi] * cos
    return y


def _appended(st):
    angle = st.pos.double()[:, None] * st.freq
    cos, sin = (angle.cos() * st.mag).float()[:, None], (angle.sin() * st.mag).float()[:, None]
    st.q_out.copy_(_turned(st.c, st.q, cos, sin))
    st.kc[st.rows] = _turned(st.c, st.k, cos, sin).to(st.kc.dtype)
    if st.vc is None:
        return [st.q_out, st.kc]
    st.vc[st.rows] = st.v
    return [st.q_out, st.kc, st.vc]


def _heads_first(q, hkv):
    """[tokens][heads][d] as [hkv][tokens * group][d] in 32 bits."""
    n, hq, d = q.shape
    return q.float().view(n, hkv, hq // hkv, d).permute(1, 0, 2, 3).reshape(hkv, n * (hq // hkv), d)


def _tokens_first(x, n):
    """Back to [tokens][heads][...]."""
    return x.unflatten(1, (n, -1)).transpose(0, 1).flatten(1, 2)


_LOWEST = torch.finfo(torch.float32).min


def _part(q, k, v, scale, hidden=None):
    """Largest logit, sum and weighted values of the rows q over the keys k; hidden [rows][keys]."""
    s = (q @ k.float().permute(1, 2, 0)).mul_(scale)
    if hidden is not None:
        s.masked_fill_(hidden, -math.inf)
    m = s.amax(-1, keepdim=True).clamp_min(_LOWEST)
    p = s.sub_(m).exp_()
    return m, p.sum(-1, keepdim=True), p @ v.float().permute(1, 0, 2)


def _joined(parts):
    m = torch.stack([p[0] for p in parts]).amax(0)
    factor = [(p[0] - m).exp() for p in parts]
    total = sum(f * p[1] for f, p in zip(factor, parts))
    o = sum(f * p[2] for f, p in zip(factor, parts))
    # a row that sees nothing: zeros, and the logarithm of zero
    return torch.where(total > 0, o / total, 0.0), torch.where(total > 0, m + total.log(), -math.inf)


def _own_hidden(lq, ls, group):
    i = torch.arange(lq, device="cuda").repeat_interleave(group)[:, None]
    return torch.arange(ls, device="cuda")[None, :] > i + ls - lq


def _shared_form(st):
    """The documents of a group for all of its rows at once, the rest for each request."""
    c, s = st.c, st.s
    group, out, lse, r = c["hq"] // c["hkv"], [], [], 0
    for per, rows in zip(s.per, st.common):
        q0, q1 = st.q_at[r], st.q_at[r + per]
        whole = _part(_heads_first(st.q[q0:q1], c["hkv"]), st.k[rows], st.v[rows], st.scale)
        for i in range(r, r + per):
            a, b, s0, s1 = st.q_at[i], st.q_at[i + 1], st.own_at[i], st.own_at[i + 1]
            q = _heads_first(st.q[a:b], c["hkv"])
            parts = [[x[:, (a - q0) * group:(b - q0) * group] for x in whole]]
            if len(st.mine[i]):
                parts.append(_part(q, st.k[st.mine[i]], st.v[st.mine[i]], st.scale))
            if s1 > s0:
                parts.append(_part(q, st.k_own[s0:s1], st.v_own[s0:s1], st.scale,
                                   _own_hidden(b - a, s1 - s0, group)))
            o, l = _joined(parts)
            out.append(_tokens_first(o, b - a))
            lse.append(_tokens_first(l, b - a)[..., 0])
        r += per
    return [torch.cat(out).to(st.q.dtype), torch.cat(lse)]


def _sparse_form(st):
    c, s = st.c, st.s
    group, out, lse, taken = c["hq"] // c["hkv"], [], [], []
    for r in range(s.batch):
        a, b, s0, s1 = st.q_at[r], st.q_at[r + 1], st.own_at[r], st.own_at[r + 1]
        means, block, lq = st.means[r], st.block[r], int(b - a)
        n = len(means)
        q = _heads_first(st.q[a:b], c["hkv"])
        # in 64 bits: what is taken must not depend on a rounding
        score = (q.double() @ means.double().permute(1, 2, 0)).unflatten(1, (lq, group)).amax(2)
        score[..., :c["first"]] = math.inf
        score[..., max(0, n - c["last"]):] = math.inf
        best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :c["blocks"]]
        best = torch.sort(best, dim=-1).values
        take = torch.zeros(score.shape, dtype=torch.bool, device="cuda").scatter_(-1, best, True)
        ids = torch.full((lq, c["hkv"], c["blocks"]), -1, dtype=torch.int32, device="cuda")
        ids[..., :best.shape[-1]] = best.transpose(0, 1)
        taken.append(ids)
        # the rows of the taken blocks, for each kv head and token
        rows = st.mine[r]
        o, l = [], []
        for i in range(lq):
            seen = take[:, i][:, block]
            most = int(min(len(rows), 64 * c["blocks"]))
            at = torch.sort(seen, dim=-1, descending=True, stable=True).indices[:, :most]
            hidden = ~torch.gather(seen, 1, at)
            head = torch.arange(c["hkv"], device="cuda")[:, None]
            k, v = st.k[rows[at], head], st.v[rows[at], head]        # [hkv][most][d]
            qi = q[:, i * group:(i + 1) * group]
            w = (qi @ k.float().transpose(1, 2)).mul_(st.scale).masked_fill_(hidden[:, None], -math.inf)
            m = w.amax(-1, keepdim=True).clamp_min(_LOWEST)
            p = w.sub_(m).exp_()
            parts = [[m, p.sum(-1, keepdim=True), p @ v.float()]]
            if s1 > s0:
                parts.append(_part(qi, st.k_own[s0:s1 - lq + i + 1], st.v_own[s0:s1 - lq + i + 1], st.scale))
            x, y = _joined(parts)
            o.append(x.flatten(0, 1))
            l.append(y.flatten())
        out.append(torch.stack(o))
        lse.append(torch.stack(l))
    return [torch.cat(out).to(st.q.dtype), torch.cat(lse), torch.cat(taken)]


# ---------------------------------------------------------------------------
# The definitions in 64 bits

def exact(case, seed):
    c, s = case, _Shape(case)
    rnd = _Draw(c, seed)
    if c["flow"] == "append":
        return _exact_append(c, s, rnd)
    k, v, q, ko, vo = _link_inputs(c, s, rnd)
    scale, group = float(np.float32(1.0 / math.sqrt(c["d"]))), c["hq"] // c["hkv"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    taken = torch.full((len(q), c["hkv"], c.get("blocks", 0)), -1, dtype=torch.int32, device="cuda")
    which = [g for g, n in enumerate(s.per) for _ in range(n)] if c["flow"] == "shared" else None
    q0 = s0 = 0
    last, kd, vd = None, None, None
    for r in range(s.batch):
        lq, ls = s.q[r], s.own[r]
        if which is None or which[r] != last:
            links = s.mine[r] if which is None else s.common[which[r]]
            take = torch.from_numpy(s.rows(links)).cuda()
            kd, vd = k[take].double().transpose(0, 1), v[take].double().transpose(0, 1)
            last = which and which[r]
        more = torch.from_numpy(s.rows(s.mine[r] if which else [])).cuda()
        for h in range(c["hkv"]):
            kh, vh = [kd[h], k[more, h].double()], [vd[h], v[more, h].double()]
            if ls:
                kh.append(ko[s0:s0 + ls, h].double())
                vh.append(vo[s0:s0 + ls, h].double())
            kh, vh = torch.cat(kh), torch.cat(vh)
            docs = len(kh) - ls
            qh = q[q0:q0 + lq, h * group:(h + 1) * group].double()
            seen = torch.ones(lq, len(kh), dtype=torch.bool, device="cuda")
            for i in range(lq):
                if ls:
                    seen[i, docs + ls - lq + i + 1:] = False
                if which is None:
                    ids = _chosen(c, s, s.mine[r], kd[h], qh[i])
                    taken[q0 + i, h, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
                    seen[i, :docs] = torch.isin(_blocks(s, s.mine[r])[1], torch.tensor(ids, device="cuda"))
            t = torch.where(seen[:, None], scale * (qh @ kh.T), -math.inf)
            total = torch.logsumexp(t, -1)
            weight = torch.exp(t - total[..., None])
            out[q0:q0 + lq, h * group:(h + 1) * group] = torch.where(seen.any(-1)[:, None, None], weight @ vh, 0.0)
            lse[q0:q0 + lq, h * group:(h + 1) * group] = total
        q0, s0 = q0 + lq, s0 + ls
    return [out, lse] if which else [out, lse, taken]


def _chosen(c, s, links, keys, q):
    """Blocks that a token's heads q [group][d] take of the keys of one kv head."""
    means, at = [], 0
    for i in links:
        part = torch.split(keys[at:at + s.lens[i]], 64)
        means += [p.mean(0, keepdim=True) for p in part]
        at += s.lens[i]
    mean = torch.cat(means).to(torch.float32).to(torch.bfloat16).double()
    score = (q @ mean.T).max(0).values.tolist()
    n = len(score)
    forced = [b < c["first"] or b >= n - c["last"] for b in range(n)]
    order = sorted(range(n), key=lambda b: (not forced[b], -score[b] if not forced[b] else 0.0, b))
    return sorted(order[:c["blocks"]])


def _exact_append(c, s, rnd):
    k_have, v_have, k, v, q, pos = _append_inputs(c, s, rnd)
    f, mag = _frequencies(c)
    z = torch.polar(torch.full((len(pos), c["rot"] // 2), mag, dtype=torch.float64, device="cuda"),
                    pos.double()[:, None] * torch.from_numpy(f).cuda())[:, None]

    def turn(x):
        y = x.double()
        part = y[..., c["rot_at"]:c["rot_at"] + c["rot"]]
        half = c["layout"] == "half"
        pairs = part.unflatten(-1, (2, -1)).transpose(-1, -2) if half else part.unflatten(-1, (-1, 2))
        turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
        y[..., c["rot_at"]:c["rot_at"] + c["rot"]] = (turned.transpose(-1, -2) if half else turned).flatten(-2)
        return y

    def chunks(have, new):
        return torch.cat([x for h, n in zip(have.split(s.have), new.split(s.add)) for x in (h.double(), n)])

    res = [turn(q), chunks(k_have, turn(k))]
    return res if v is None else res + [chunks(v_have, v.double())]
