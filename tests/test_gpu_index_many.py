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
