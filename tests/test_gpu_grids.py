"""Calls whose workgroups pass the 2^32 threads of one launch: many requests, one of them long,
since every request has room for the longest one's row blocks. Every request links the same
chunk, so that one product per kv head gives the reference, in 64 bits on the GPU.

Tolerances as derived in fp4_model.py and test_gpu_far_logits.py (bf16: both the widest);
fp32 stores round nothing to fewer bits: products, sums, exponentials and the division are off by
a few 2^-24 of their size, e per probability and as much for each of the rest."""
import numpy as np
import pytest
import torch

import fp4_model as M
from paper_2602_01519_amd import pic

pytestmark = pytest.mark.gpu

# kind, dtype, d_k, d_v, query heads, kv heads, tokens of the long request
CASES = {
    "fp4": (pic.GQA, pic.FP4, 64, 64, 32, 8, 32768),
    "fp4_128": (pic.GQA, pic.FP4, 128, 128, 32, 8, 32768),
    "fp4_longer": (pic.GQA, pic.FP4, 64, 64, 32, 8, 131072),
    "d128": (pic.GQA, pic.BF16, 128, 128, 32, 8, 131072),
    "stream": (pic.GQA, pic.BF16, 64, 64, 32, 8, 262144),
    "stream_fp32": (pic.GQA, pic.F32, 32, 32, 32, 8, 131072),
    "vector": (pic.GQA, pic.BF16, 96, 96, 32, 8, 16384),
    "mla": (pic.MLA, pic.BF16, 576, 512, 16, 1, 131072),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_one_long_request_among_many_short_ones(name):
    kind, dtype, d, dv, hq, hkv, long = CASES[name]
    mla, n, group = kind == pic.MLA, 70, hq // hkv
    t = torch.float32 if dtype == pic.F32 else torch.bfloat16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(t)  # noqa: E731
    k = draw(n, hkv, d)
    v = None if mla else draw(n, hkv, dv)
    lens = [1] * 256 + [long] + [1] * 256
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q = draw(int(off[-1]), hq, d)
    out = torch.full((len(q), hq, dv), 7.0, dtype=t, device="cuda")
    lse = torch.full((len(q), hq), 5.0, dtype=torch.float32, device="cuda")
    scale = float(np.float32(d ** -0.5))
    st = torch.cuda.current_stream().cuda_stream
    print(name, flush=True)
    with pic.Store(kind, dtype, hkv, d, dv, 128) as store:
        store.put(1, n, k, v, st)
        pic.link_attn(store, list(range(len(lens) + 1)), [1] * len(lens), off, None, hq, q, None, None, scale, out,
                      lse, stream=st)
        torch.cuda.synchronize()
    kept = (lambda x: torch.from_numpy(M.stored(x.double().cpu().numpy())).cuda()) if dtype == pic.FP4 else \
        (lambda x: x.double())
    kk = kept(k)
    vv = kk[..., :dv] if mla else kept(v)
    u = 2.0 ** -24
    half = 0.0 if dtype == pic.F32 else 2.0 ** -8
    for h in range(hkv):
        kt, vh = kk[:, h].T.contiguous(), vv[:, h].contiguous()
        heads = slice(h * group, (h + 1) * group)
        for a in range(0, len(q), 1 << 14):
            rows = q[a:a + (1 << 14), heads].reshape(-1, d).double()
            s = scale * (rows @ kt)
            top = s.amax(1, keepdim=True)
            p = torch.exp(s - top)
            w = p / p.sum(1, keepdim=True)
            ref, z = w @ vh, (top + torch.log(p.sum(1, keepdim=True)))[:, 0]
            e = u * (d * scale * (rows.abs() @ kt.abs()).amax(1) + 4 * s.abs().amax(1) + n + 16)
            tol = 2.05 * half * ref.abs() + (2.05 * half + 8 * e[:, None]) * (w @ vh.abs())
            o, l = out[a:a + (1 << 14), heads].reshape(-1, dv).double(), lse[a:a + (1 << 14), heads].reshape(-1).double()
            assert bool(((o - ref).abs() <= tol).all()), f"tokens from {a}, kv head {h}"
            assert bool(((l - z).abs() <= 1.01 * half + e + 4 * u * z.abs()).all()), f"tokens from {a}, kv head {h}"


def test_a_batch_of_many_requests_in_pieces():
    """70,000 requests of one token, each cut in two: items, and requests of the combine."""
    b, d, n = 70000, 64, 70
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    k, v, q = draw(n, 1, d), draw(n, 1, d), draw(b, 2, d)
    out = torch.full_like(q, 7.0)
    st = torch.cuda.current_stream().cuda_stream
    with pic.Store(pic.GQA, pic.FP4, 1, d, d, 128) as store:
        store.put(1, n, k, v, st)
        at = np.arange(b + 1, dtype=np.int32)
        pic.link_decode(store, at, np.ones(b, np.uint64), at, None, 2, q, None, None, 0.125, out, None, num_splits=2,
                        stream=st)
        torch.cuda.synchronize()
    kk, vv = (torch.from_numpy(M.stored(x[:, 0].double().cpu().numpy())).cuda() for x in (k, v))
    rows = q.double().reshape(-1, d)
    w = torch.softmax(0.125 * (rows @ kk.T.contiguous()), 1)
    e = 2.0 ** -24 * (d * 0.125 * (rows.abs() @ kk.abs().T.contiguous()).amax(1) * 5 + n + 16)
    ref = w @ vv
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 4 * e[:, None]) * (w @ vv.abs())
    assert bool(((out.double().reshape(-1, d) - ref).abs() <= tol).all())


@pytest.mark.parametrize("links", [1, 40])
def test_one_request_of_more_than_a_launch(links):
    """2^29 query rows of one request (a call has at most 2^30 - 1) in blocks of 16: refused on the
    host, before any tensor is looked at (40 links: not a small call)."""
    x = torch.zeros(64, 1, 8, dtype=torch.bfloat16, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    with pic.Store(pic.GQA, pic.BF16, 1, 8, 8, 64) as store:
        store.put(1, 64, x, x, st)
        with pytest.raises(pic.PicError) as e:
            pic.link_attn(store, [0, links], [1] * links, [0, 1 << 19], None, 1024, x, None, None, 1.0, x, None, stream=st)
        assert e.value.status == pic.ERR_UNSUPPORTED
