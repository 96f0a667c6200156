"""One update of a block index over more than 2^32 threads' worth of pages, chunks and layers."""
import numpy as np
import pytest
import torch

import link_model as L
from paper_2602_01519_amd import pic
from test_gpu_sparse import chosen, summaries

pytestmark = pytest.mark.gpu


def test_long_chunk_among_many_in_many_layers():
    hkv, d, layers, pages, n = 8, 64, 32, 700, 8
    assert pages * 96 * hkv * layers * 256 > 2 ** 32        # (96 pieces a launch, 256 threads a page)
    tokens = pages * 64 - 9
    gen = torch.Generator("cuda").manual_seed(3)
    with pic.Store(pic.GQA, pic.BF16, hkv, d, d, 64 * (pages + 95), n_layers=layers) as store:
        k = torch.randn(layers, tokens, hkv, d, device="cuda", generator=gen, dtype=torch.float32).bfloat16()
        store.put(0, tokens, k, torch.zeros_like(k), L.stream())
        short = torch.randn(layers, 95, hkv, d, device="cuda", generator=gen).bfloat16()
        for i in range(95):
            x = short[:, i:i + 1].contiguous()
            store.put(1 + i, 1, x, x, L.stream())
        with pic.BlockIndex(store) as index:
            index.update(range(96), stream=L.stream())
            q = torch.randn(1, hkv, d, device="cuda", generator=gen).bfloat16()
            for layer in (0, 17, layers - 1):
                out, taken = torch.zeros_like(q), torch.full((1, hkv, n), -9, dtype=torch.int32, device="cuda")
                pic.link_sparse(index, [0, 3], [5, 0, 95], [0, 1], None, hkv, n, q, None, None, 0.125, out, blocks=taken,
                                stream=L.stream(), layer=layer)
                torch.cuda.synchronize()
                keys = torch.cat([short[layer, 4:5], k[layer], short[layer, 94:95]])
                means, _ = summaries(keys, [1, tokens, 1])
                want = [chosen(means[:, h], q[0, h:h + 1], n, 0, 0) for h in range(hkv)]
                assert taken[0].tolist() == want, layer


@pytest.mark.parametrize("dtype,d", [(pic.BF16, 64), (pic.F32, 128)])
def test_layers_that_hold_differently_many_tokens(dtype, d):
    """A growing chunk behind a document, each layer with rows of its own number: blocks and outputs of both."""
    rng = np.random.default_rng(d)
    hkv, hq, n, scale = 2, 6, 3, 0.125
    with pic.Store(pic.GQA, dtype, hkv, d, d, 64 * 20, n_layers=2) as store, pic.BlockIndex(store) as index:
        doc = [L.draw(rng, dtype, 2, 130, hkv, d) for _ in range(2)]
        store.put(1, 130, *doc, L.stream())
        store.open(2, 700)
        held = [[x[layer] for x in doc] for layer in range(2)]
        for counts in ([150, 300], [1, 0], [0, 21], [63, 64]):
            for layer, m in enumerate(counts):
                k, v = (L.draw(rng, dtype, m, hkv, d) for _ in range(2))
                store.append([2], [0, m], k, v, stream=L.stream(), layer=layer)
                held[layer] = [torch.cat([a, b]) for a, b in zip(held[layer], (k, v))]
            index.update([1, 2], stream=L.stream())
            q = L.draw(rng, dtype, 1, hq, d)
            for layer in range(2):
                k, v = held[layer]
                out, lse = torch.full_like(q, 7.0), torch.zeros(1, hq, dtype=torch.float32, device="cuda")
                taken = torch.full((1, hkv, n), -9, dtype=torch.int32, device="cuda")
                pic.link_sparse(index, [0, 2], [1, 2], [0, 1], None, hq, n, q, None, None, scale, out, lse, keep_last=1,
                                blocks=taken, stream=L.stream(), layer=layer)
                torch.cuda.synchronize()
                means, block = summaries(k, [130, len(k) - 130])
                refs = []
                for h in range(hkv):
                    want = chosen(means[:, h], q[0, 3 * h:3 * h + 3], n, 0, 1)
                    assert taken[0, h].tolist() == want, (counts, layer, h)
                    rows = torch.isin(block, torch.tensor(want, device="cuda"))
                    refs.append(L.attend(q[:, 3 * h:3 * h + 3], k[rows, h:h + 1], v[rows, h:h + 1], scale))
                L.check(dtype, out, lse, *(torch.cat(x, 1) for x in zip(*refs)))
