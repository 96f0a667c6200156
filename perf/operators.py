"""The 4-bit chunk cache, link attention over it, and rotary positions, as cases for
performance measurement.

  put     a document's caches are put into a store that holds them in 4 bits, read back
          and removed
  link    prefill-shaped link attention of a batch over such a store (pic_link_attn)
  decode  one decode step of a batch over it (a link plan, or pic_link_decode)
  rope    rotary positions of a batch's queries and keys, or the gradient of that

`run` computes the plain form (elementary torch operations) unless `own` is set; then it
makes the calls of paper_2602_01519_amd.pic. A case is a dict of plain values; its ragged
sizes come from its "shape" number, tensor values from the seed.

The 4-bit format: a row (one token, one head) is cut into blocks of 32; a block holds the
numbers 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, times 2^e, where e is the smallest exponent
(from -126 to 125) with max|x| < 7 * 2^e. Elements are rounded to the nearest, ties to the even code.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False


def _case(name=None, **kw):
    c = dict(kw)
    if name is not None:
        c = {"name": name, **c}
    return c


def _put(name=None, *, tokens, hkv, d, layers):
    return _case(name, flow="put", tokens=tokens, hkv=hkv, d=d, layers=layers)


def _link(name=None, *, flow="link", hq, hkv, d, batch, chunks, len_lo, len_hi, links_lo, links_hi,
          q_lo, q_hi, own_extra=0, own_kv=True, disjoint=False, starts=False, limits=False,
          plan=False, shape=1):
    return _case(name, flow=flow, hq=hq, hkv=hkv, d=d, batch=batch, chunks=chunks, len_lo=len_lo,
                 len_hi=len_hi, links_lo=links_lo, links_hi=links_hi, q_lo=q_lo, q_hi=q_hi,
                 own_extra=own_extra, own_kv=own_kv, disjoint=disjoint, starts=starts,
                 limits=limits, plan=plan, shape=shape)


def _rope(name=None, *, tokens, hq, hk, width, rot_at, rot, dtype="bf16", layout="half",
          scaling="none", theta=10000.0, factor=1.0, far=4096, fused=False, transposed=False):
    return _case(name, flow="rope", tokens=tokens, hq=hq, hk=hk, width=width, rot_at=rot_at,
                 rot=rot, dtype=dtype, layout=layout, scaling=scaling, theta=theta, factor=factor,
                 far=far, fused=fused, transposed=transposed)


def listed():
    return [
        # One short document enters the cache while a user waits: launches.
        _put("put_short", tokens=200, hkv=8, d=128, layers=1),
        # A long document, all of its eight cross-attention layers.
        _put("put_long", tokens=7000, hkv=8, d=128, layers=8),
        # One question of a few dozen tokens over ten ragged documents: the time to first
        # token of a single interactive user.
        _link("question", hq=32, hkv=8, d=128, batch=1, chunks=16, len_lo=200, len_hi=1100,
              links_lo=10, links_hi=10, q_lo=37, q_hi=37, shape=2),
        # Batched prefill with the head shape of an 8B GQA backbone, shared documents.
        _link("llama_prefill", hq=32, hkv=8, d=128, batch=8, chunks=64, len_lo=512, len_hi=512,
              links_lo=10, links_hi=10, q_lo=256, q_hi=256, shape=4),
        # The largest: 16 requests with 8..20 documents of 1024 tokens, 512 query tokens.
        _link("long_rag", hq=32, hkv=8, d=128, batch=16, chunks=256, len_lo=1024, len_hi=1024,
              links_lo=8, links_hi=20, q_lo=512, q_hi=512, shape=5),
        # 64-wide heads, ragged requests whose links skip the recomputed first tokens.
        _link("narrow_heads", hq=32, hkv=8, d=64, batch=8, chunks=64, len_lo=100, len_hi=1000,
              links_lo=4, links_hi=12, q_lo=30, q_hi=300, starts=True, shape=11),
        # One decode step of one user over a few documents, planned once: latency.
        _link("decode_one", flow="decode", hq=32, hkv=8, d=128, batch=1, chunks=8, len_lo=150,
              len_hi=900, links_lo=5, links_hi=5, q_lo=1, q_hi=1, own_extra=40, plan=True,
              shape=7),
        # One decode step of a full batch, 16 private documents each: bound by the cache's bytes.
        _link("decode_batch", flow="decode", hq=32, hkv=8, d=128, batch=64, chunks=1024,
              len_lo=1024, len_hi=1024, links_lo=16, links_hi=16, q_lo=1, q_hi=1, disjoint=True,
              own_extra=127, plan=True, shape=6),
        # A few tokens per request are checked at once, 64-wide heads, odd head counts.
        _link("decode_tokens", flow="decode", hq=24, hkv=6, d=64, batch=12, chunks=80, len_lo=90,
              len_hi=1000, links_lo=3, links_hi=9, q_lo=1, q_hi=4, own_extra=33, shape=9),
        # Positions of one decode step's queries and keys.
        _rope("rope_step", tokens=64, hq=32, hk=8, width=128, rot_at=0, rot=128, theta=500000.0,
              scaling="banded", factor=8.0, far=130000, fused=True),
        # Positions of a prefill batch, queries and keys inside the fused projection's output.
        _rope("rope_prefill", tokens=8192, hq=32, hk=8, width=128, rot_at=0, rot=128,
              theta=500000.0, scaling="banded", factor=8.0, far=130000, fused=True),
        # Gradient through the rotated part of MLA-shaped heads, stretched to long contexts.
        _rope("rope_grad", tokens=4099, hq=16, hk=1, width=192, rot_at=128, rot=64, dtype="f32",
              layout="interleaved", scaling="yarn", factor=40.0, far=160000, transposed=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _span(rng, lo, hi):
    return sorted((_log_int(rng, lo, hi), _log_int(rng, lo, hi)))


def draw(rng):
    """One more case of the listed ranges, no more work than the largest of its flow."""
    flow = rng.choice(["put", "link", "link", "decode", "decode", "rope"])
    most = {}
    for c in listed():
        w = work(c)
        for k in w:
            most[c["flow"], k] = max(w[k], most.get((c["flow"], k), 0.0))
    while True:
        hkv = rng.choice([1, 2, 3, 4, 6, 8])
        hq = hkv * rng.choice([1, 2, 3, 4, 5, 8])
        d = rng.choice([64, 128, 128])
        if flow == "put":
            c = _put(tokens=_log_int(rng, 1, 12000), hkv=hkv, d=d, layers=rng.randint(1, 8))
        elif flow == "rope":
            rot = 2 * rng.randint(4, 64)
            rest = 8 * rng.randint(0, 16)
            c = _rope(tokens=_log_int(rng, 1, 8192), hq=hq, hk=hkv, width=rot + rest,
                      rot_at=rng.choice([0, rest]), rot=rot, dtype=rng.choice(["bf16", "bf16", "f32"]),
                      layout=rng.choice(["half", "interleaved"]),
                      scaling=rng.choice(["none", "linear", "banded", "yarn"]),
                      theta=rng.choice([10000.0, 500000.0]), factor=float(rng.choice([2, 8, 40])),
                      far=_log_int(rng, 16, 1000000), fused=rng.random() < 0.5,
                      transposed=rng.random() < 0.5)
        else:
            len_lo, len_hi = _span(rng, 1, 1100)
            links_lo, links_hi = _span(rng, 1, 20)
            q_lo, q_hi = _span(rng, 1, 512 if flow == "link" else 6)
            batch = _log_int(rng, 1, 16 if flow == "link" else 64)
            disjoint = rng.random() < 0.4
            own_kv = rng.random() < 0.8
            c = _link(flow=flow, hq=hq, hkv=hkv, d=d, batch=batch, len_lo=len_lo, len_hi=len_hi,
                      links_lo=links_lo, links_hi=links_hi, q_lo=q_lo, q_hi=q_hi,
                      own_extra=_log_int(rng, 1, 200), own_kv=own_kv, disjoint=disjoint,
                      chunks=batch * links_hi if disjoint else links_hi + _log_int(rng, 1, 200),
                      starts=rng.random() < 0.3, limits=flow == "link" and rng.random() < 0.25,
                      plan=rng.random() < 0.5, shape=rng.randrange(1 << 20))
        w = work(c)
        if all(w[k] <= most[flow, k] for k in w) and (flow in ("put", "rope") or w["flops"] > 1e6):
            return c


# ---------------------------------------------------------------------------
# Shapes of a case

class _Shape:
    """Chunk lengths, links and token counts of a link or decode case."""

    def __init__(self, c):
        r = random.Random(c["shape"])
        self.lens = [r.randint(c["len_lo"], c["len_hi"]) for _ in range(c["chunks"])]
        counts = [r.randint(c["links_lo"], c["links_hi"]) for _ in range(c["batch"])]
        if c["disjoint"]:
            perm = list(range(c["chunks"]))
            r.shuffle(perm)
            self.links = [[perm.pop() for _ in range(n)] for n in counts]
        else:
            self.links = [r.sample(range(c["chunks"]), n) for n in counts]
        self.q = [r.randint(c["q_lo"], c["q_hi"]) for _ in range(c["batch"])]
        self.own = [n + c["own_extra"] if c["own_kv"] else 0 for n in self.q]
        self.start = [64 if c["starts"] and n > 64 else 0 for n in self.lens]
        self.used = sorted({i for l in self.links for i in l})
        self.doc = [sum(self.lens[i] - self.start[i] for i in l) for l in self.links]
        # with limits, query i of a request sees the linked rows up to a position of its own
        self.seen = [[r.randint(0, n) if c["limits"] else n for _ in range(m)]
                     for n, m in zip(self.doc, self.q)]


def _offsets(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def _chunk_id(i):
    return 0x5851F42D4C957F2D * (i + 1) & 0x7FFFFFFFFFFFFFFF


def work(case):
    """Bytes and operations of one pass: inputs read once, outputs written once, only the
    pairs that see each other. 4-bit caches: 17 bytes per 32 elements."""
    c = case
    if c["flow"] == "put":
        n = 2 * c["layers"] * c["tokens"] * c["hkv"] * c["d"]
        # put: bf16 in, 4 bits out; read back: 4 bits in, bf16 out
        return {"bytes": 2.0 * n * (2 + 17 / 32), "flops": 4.0 * n}
    if c["flow"] == "rope":
        es = 4 if c["dtype"] == "f32" else 2
        rows = c["tokens"] * (c["hq"] + c["hk"])
        return {"bytes": 2.0 * es * rows * c["width"] + 4.0 * c["tokens"],
                "flops": 3.0 * rows * c["rot"]}
    s = _Shape(c)
    tq, row = sum(s.q), c["hkv"] * 2 * c["d"]
    bytes_ = sum(s.lens[i] - s.start[i] for i in s.used) * row * 17 / 32 + sum(s.own) * row * 2 \
        + tq * c["hq"] * (4 * c["d"] + 4)
    pairs = 0
    for r in range(c["batch"]):
        pairs += sum(s.seen[r])
        if s.own[r]:
            pairs += sum(i + 1 + s.own[r] - s.q[r] for i in range(s.q[r]))
    return {"bytes": float(bytes_), "flops": float(pairs * c["hq"] * 4 * c["d"])}


# ---------------------------------------------------------------------------
# Inputs

class _Draw:
    """Seeded N(0, 1) tensors, one after another."""

    def __init__(self, c, seed, dtype=torch.bfloat16):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed * 1000003 + c.get("shape", 0))
        self.dtype = dtype

    def __call__(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda",
                           dtype=torch.float32).to(self.dtype)


class _State:
    pass


def _frequencies(c):
    """Angle per position of every rotated pair, in 64 bits, and the factor of cos and sin."""
    half = c["rot"] // 2
    f = c["theta"] ** (-np.arange(half, dtype=np.float64) / half)
    if c["scaling"] == "linear":
        return f / c["factor"], 1.0
    if c["scaling"] == "banded":
        # slow turns (fewer than _LOW in the original length) are stretched, fast ones
        # (more than _HIGH) kept, a linear blend between
        keep = np.clip((_LENGTH * f / (2 * np.pi) - _LOW) / (_HIGH - _LOW), 0.0, 1.0)
        return f * (keep + (1.0 - keep) / c["factor"]), 1.0
    if c["scaling"] == "yarn":
        # the same by the pair's index, between the pairs that turn _FAST and _SLOW times
        at = lambda turns: half * math.log(_LENGTH / (turns * 2 * math.pi)) / math.log(c["theta"])  # noqa: E731
        lo = max(math.floor(at(_FAST)), 0)
        hi = min(math.ceil(at(_SLOW)), c["rot"] - 1)
        ramp = np.clip((np.arange(half) - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return f * ((1.0 - ramp) + ramp / c["factor"]), 0.1 * math.log(c["factor"]) + 1.0
    return f, 1.0


_LENGTH, _LOW, _HIGH, _FAST, _SLOW = 4096, 1.0, 4.0, 32.0, 1.0


def _rope_inputs(c, seed):
    rnd = _Draw(c, seed, torch.float32 if c["dtype"] == "f32" else torch.bfloat16)
    t, hq, hk, w = c["tokens"], c["hq"], c["hk"], c["width"]
    if c["fused"]:                      # slices of [q heads | k heads | v heads] rows
        x = rnd(t, hq + 2 * hk, w)
        xs = [x[:, :hq], x[:, hq:hq + hk]]
    else:
        xs = [rnd(t, hq, w), rnd(t, hk, w)]
    pos = torch.randint(0, c["far"], (t,), generator=rnd.gen, device="cuda", dtype=torch.int32)
    return xs, pos


def _stream():
    return torch.cuda.current_stream().cuda_stream


def prepare(case, seed):
    c = case
    st = _State()
    st.c = c
    if own:
        from paper_2602_01519_amd import pic
    if c["flow"] == "rope":
        st.x, st.pos = _rope_inputs(c, seed)
        st.out = [torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in st.x]
        f, st.mag = _frequencies(c)
        st.freq = torch.from_numpy(f).cuda()
        if own:
            st.rope = pic.Rope(pic.F32 if c["dtype"] == "f32" else pic.BF16,
                               pic.ROPE_HALF if c["layout"] == "half" else pic.ROPE_INTERLEAVED,
                               c["width"], c["rot_at"], c["rot"], theta=c["theta"],
                               scaling={"none": pic.ROPE_PLAIN, "linear": pic.ROPE_LINEAR,
                                        "banded": pic.ROPE_BANDED, "yarn": pic.ROPE_YARN}[c["scaling"]],
                               factor=c["factor"], original_len=_LENGTH, band_low=_LOW,
                               band_high=_HIGH, turns_fast=_FAST, turns_slow=_SLOW,
                               magnitude=st.mag)
            st.tensors = [(x, y, x.shape[1], x.stride(0), 0) for x, y in zip(st.x, st.out)]
        return st
    rnd = _Draw(c, seed)
    if c["flow"] == "put":
        shape = (c["layers"], c["tokens"], c["hkv"], c["d"])
        st.k, st.v = rnd(*shape), rnd(*shape)
        if own:
            # room for the documents whose removal is still pending
            st.store = pic.Store(pic.GQA, pic.FP4, c["hkv"], c["d"], c["d"],
                                 4 * ((c["tokens"] + 63) // 64 * 64), n_layers=c["layers"])
            st.k_out, st.v_out = torch.empty_like(st.k), torch.empty_like(st.v)
        return st
    s = st.s = _Shape(c)
    lens = [s.lens[i] for i in s.used]
    at = np.concatenate([[0], np.cumsum(lens)])
    k, v = rnd(int(at[-1]), c["hkv"], c["d"]), rnd(int(at[-1]), c["hkv"], c["d"])
    tq, ts = sum(s.q), sum(s.own)
    st.q = rnd(tq, c["hq"], c["d"])
    st.k_own = rnd(ts, c["hkv"], c["d"]) if c["own_kv"] else None
    st.v_own = rnd(ts, c["hkv"], c["d"]) if c["own_kv"] else None
    st.scale = float(np.float32(1.0 / math.sqrt(c["d"])))
    st.limits = np.array([n for l in s.seen for n in l], dtype=np.int32) if c["limits"] else None
    if own:
        st.store = pic.Store(pic.GQA, pic.FP4, c["hkv"], c["d"], c["d"],
                             sum((n + 63) // 64 * 64 for n in lens))
        for i, a, n in zip(s.used, at, lens):
            st.store.put(_chunk_id(i), n, k[a:a + n], v[a:a + n], _stream())
        index = [i for l in s.links for i in l]
        st.offsets = _offsets([len(l) for l in s.links])
        st.ids = np.array([_chunk_id(i) for i in index], dtype=np.uint64)
        st.q_offsets = _offsets(s.q)
        st.own_offsets = _offsets(s.own) if c["own_kv"] else None
        st.starts = np.array([s.start[i] for i in index], dtype=np.int32) if c["starts"] else None
        st.out = torch.empty_like(st.q)
        st.lse = torch.empty(tq, c["hq"], dtype=torch.float32, device="cuda")
        if c["plan"]:
            st.plan = pic.LinkPlan(st.store, st.offsets, st.ids, st.q_offsets, st.own_offsets,
                                   c["hq"], mode=pic.DECODE if c["flow"] == "decode" else pic.PREFILL,
                                   chunk_starts=st.starts, q_doc_limits=st.limits)
        torch.cuda.synchronize()        # k and v are freed here
        return st
    st.kc, st.vc = _encoded(k), _encoded(v)
    # cache rows of each request, in link order
    first = dict(zip(s.used, at))
    st.rows = [torch.from_numpy(np.concatenate(
        [np.arange(first[i] + s.start[i], first[i] + s.lens[i]) for i in l])).cuda() for l in s.links]
    st.q_at, st.own_at = _offsets(s.q), _offsets(s.own)
    # linked rows that each query sees
    st.seen = [torch.tensor(n, device="cuda") for n in s.seen]
    return st


# ---------------------------------------------------------------------------
# One pass

def run(st):
    if own:
        return _run_own(st)
    flow = st.c["flow"]
    if flow == "rope":
        return [_rotated(st.c, x, st.pos, st.freq, st.mag) for x in st.x]
    if flow == "put":
        return [_decoded(*_encode(x)).to(torch.bfloat16) for x in (st.k, st.v)]
    return _linked(st)


def _run_own(st):
    from paper_2602_01519_amd import pic
    c, stream = st.c, _stream()
    if c["flow"] == "rope":
        st.rope.apply(c["tokens"], st.pos, st.tensors, transposed=c["transposed"], stream=stream)
        return st.out
    if c["flow"] == "put":
        st.store.put(1, c["tokens"], st.k, st.v, stream)
        for l in range(c["layers"]):
            pic.debug_gather(st.store, [1], st.k_out[l], st.v_out[l], stream, layer=l)
        st.store.remove(1, stream)
        return [st.k_out, st.v_out]
    if c["plan"]:
        st.plan.run(0, st.q, st.k_own, st.v_own, st.scale, st.out, st.lse, stream)
    else:
        link = pic.link_decode if c["flow"] == "decode" else pic.link_attn
        link(st.store, st.offsets, st.ids, st.q_offsets, st.own_offsets, c["hq"], st.q, st.k_own,
             st.v_own, st.scale, st.out, st.lse, stream=stream, chunk_starts=st.starts,
             q_doc_limits=st.limits)
    return [st.out, st.lse]


# ---------------------------------------------------------------------------
# The plain forms

_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _encode(x):
    """Codes 0..15 (sign, then the index of _VALUES) and exponents of blocks of 32."""
    b = x.float().unflatten(-1, (-1, 32))
    frac, e = torch.frexp(b.abs().amax(-1, keepdim=True))       # max = frac * 2^e, frac < 1
    e = (e - 3 + (frac >= 0.875)).clamp(-126, 125)
    y = torch.ldexp(b, -e).abs()
    # borders between neighbours; a value on a border goes to the even code
    code = (y > 0.25).int() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)
    return (code + 8 * torch.signbit(b)).to(torch.uint8).flatten(-2), e.squeeze(-1)


def _decoded(code, e):
    """The values that codes and block exponents stand for, in 32 bits."""
    table = torch.tensor(_VALUES + [-x for x in _VALUES], device=code.device)
    return torch.ldexp(table[code.int()].unflatten(-1, (-1, 32)), e.int().unsqueeze(-1)).flatten(-2)


def _encoded(x):
    """x as a program keeps it: two codes in a byte, exponents in bytes. In slices, since the
    values in between take many times the room."""
    parts = [_encode(p) for p in x.split(1 << 16)]
    code = torch.cat([p[:, :, 0::2] | p[:, :, 1::2] << 4 for p, _ in parts])
    return code, torch.cat([e.to(torch.int8) for _, e in parts])


def _cached(cache, rows):
    """Cache rows [n][heads][width] in 32 bits."""
    code, e = cache[0][rows], cache[1][rows]
    return _decoded(torch.stack([code & 15, code >> 4], -1).flatten(-2), e)


def _linked(st):
    c = st.c
    hkv, group, d = c["hkv"], c["hq"] // c["hkv"], c["d"]
    out, lse = [], []
    for r in range(c["batch"]):
        q0, q1, s0, s1 = st.q_at[r], st.q_at[r + 1], st.own_at[r], st.own_at[r + 1]
        lq, ls = int(q1 - q0), int(s1 - s0)
        k, v = _cached(st.kc, st.rows[r]), _cached(st.vc, st.rows[r])
        doc = k.shape[0]
        if ls:
            k, v = torch.cat([k, st.k_own[s0:s1].float()]), torch.cat([v, st.v_own[s0:s1].float()])
        q = st.q[q0:q1].float().view(lq, hkv, group, d).permute(1, 0, 2, 3).reshape(hkv, lq * group, d)
        s = (q @ k.permute(1, 2, 0)).mul_(st.scale).view(hkv, lq, group, -1)
        i = torch.arange(lq, device="cuda")[:, None]
        j = torch.arange(doc + ls, device="cuda")[None, :]
        hidden = torch.where(j < doc, j >= st.seen[r][:, None], j - doc > i + ls - lq)
        s.masked_fill_(hidden[None, :, None, :], -math.inf)
        m = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
        p = s.sub_(m).exp_()
        total = p.sum(-1, keepdim=True)
        o = (p.view(hkv, lq * group, -1) @ v.permute(1, 0, 2)).view(hkv, lq, group, d)
        # a row that sees nothing: zeros, and the logarithm of zero
        o = torch.where(total > 0, o / total, 0.0)
        out.append(o.permute(1, 0, 2, 3).reshape(lq, c["hq"], d))
        lse.append(torch.where(total > 0, m + total.log(), -math.inf).permute(1, 0, 2, 3).reshape(lq, c["hq"]))
    return [torch.cat(out).to(torch.bfloat16), torch.cat(lse)]


def _rotated(c, x, pos, freq, mag):
    """x with the pairs of its rotated part turned by pos * freq (back, for the gradient)."""
    angle = pos.double()[:, None] * freq
    cos, sin = (angle.cos() * mag).float()[:, None], (angle.sin() * mag).float()[:, None]
    if c["transposed"]:
        sin = -sin
    x = x.float()
    a, r = c["rot_at"], c["rot"]
    y = x.clone()
    if c["layout"] == "half":
        lo, hi = slice(a, a + r // 2), slice(a + r // 2, a + r)
    else:
        lo, hi = slice(a, a + r, 2), slice(a + 1, a + r, 2)
    y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
    y[..., hi] = x[..., lo] * sin + x[..., hi] * cos
    return y.to(torch.float32 if c["dtype"] == "f32" else torch.bfloat16)


# ---------------------------------------------------------------------------
# The definitions in 64 bits

def _nearest4(x):
    """x in 64 bits, every block of 32 on its grid: the exponent by search, the value by distance."""
    b = x.double().reshape(*x.shape[:-1], -1, 32)
    top = b.abs().max(-1, keepdim=True).values
    step = torch.full_like(top, 2.0 ** -126)
    log = torch.floor(torch.log2(torch.where(top > 0, top / 7, 1.0)))
    for up in (-1, 0, 1, 2):            # the smallest power of two that keeps top below 7 of it
        t = torch.exp2((log + up).clamp(-126, 125))
        ok = (top > 0) & (step * 7 <= top) & (top < 7 * t)
        step = torch.where(ok, t, step)
    # even codes first, so that the first of two equally near ones is the even one
    grid = torch.tensor([0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0], device=x.device, dtype=torch.float64)
    y = b.abs() / step
    best, near = torch.zeros_like(y), torch.full_like(y, math.inf)
    for g in grid:
        far = (y - g).abs()
        best, near = torch.where(far < near, g, best), torch.minimum(far, near)
    return (torch.copysign(best, b) * step).reshape(x.shape)


def exact(case, seed):
    c = case
    if c["flow"] == "rope":
        xs, pos = _rope_inputs(c, seed)
        f, mag = _frequencies(c)
        z = torch.polar(torch.full((c["tokens"], c["rot"] // 2), mag, dtype=torch.float64, device="cuda"),
                        pos.double()[:, None] * torch.from_numpy(f).cuda())
        z = (z.conj() if c["transposed"] else z)[:, None]
        out = []
        for x in xs:
            y = x.double()
            part = y[..., c["rot_at"]:c["rot_at"] + c["rot"]]
            half = c["layout"] == "half"
            pairs = part.unflatten(-1, (2, -1)).transpose(-1, -2) if half else part.unflatten(-1, (-1, 2))
            turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
            y[..., c["rot_at"]:c["rot_at"] + c["rot"]] = \
                (turned.transpose(-1, -2) if half else turned).flatten(-2)
            out.append(y)
        return out
    rnd = _Draw(c, seed)
    if c["flow"] == "put":
        shape = (c["layers"], c["tokens"], c["hkv"], c["d"])
        k, v = rnd(*shape), rnd(*shape)
        return [torch.cat([_nearest4(l)[None] for l in x]) for x in (k, v)]
    s = _Shape(c)
    lens = [s.lens[i] for i in s.used]
    at = dict(zip(s.used, np.concatenate([[0], np.cumsum(lens)])))
    k, v = rnd(sum(lens), c["hkv"], c["d"]), rnd(sum(lens), c["hkv"], c["d"])
    q = rnd(sum(s.q), c["hq"], c["d"])
    if c["own_kv"]:
        ko, vo = rnd(sum(s.own), c["hkv"], c["d"]), rnd(sum(s.own), c["hkv"], c["d"])
    scale = float(np.float32(1.0 / math.sqrt(c["d"])))
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    group, q0, s0 = c["hq"] // c["hkv"], 0, 0
    for r, links in enumerate(s.links):
        lq, ls = s.q[r], s.own[r]
        take = torch.cat([torch.arange(at[i] + s.start[i], at[i] + s.lens[i]) for i in links]).cuda()
        doc = len(take)
        seen = torch.zeros(lq, doc + ls, dtype=torch.bool, device="cuda")
        for i in range(lq):
            seen[i, :s.seen[r][i]] = True
            seen[i, doc:doc + i + 1 + ls - lq] = True
        for h in range(c["hkv"]):
            kh, vh = _nearest4(k[take, h]), _nearest4(v[take, h])
            if ls:
                kh, vh = torch.cat([kh, ko[s0:s0 + ls, h].double()]), torch.cat([vh, vo[s0:s0 + ls, h].double()])
            for g in range(h * group, (h + 1) * group):
                t = torch.where(seen, scale * (q[q0:q0 + lq, g].double() @ kh.T), -math.inf)
                total = torch.logsumexp(t, -1)
                weight = torch.exp(t - total[:, None])
                out[q0:q0 + lq, g] = torch.where(seen.any(-1)[:, None], weight @ vh, 0.0)
                lse[q0:q0 + lq, g] = total
        q0, s0 = q0 + lq, s0 + ls
    return [out, lse]
