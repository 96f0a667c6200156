"""Grown chunks handed over to another process: the rows that every layer holds, linked there."""
import multiprocessing as mp

import numpy as np
import pytest
import torch

import append_ipc_child
import link_model as L
from paper_2602_01519_amd import pic
from test_gpu_append import Chunks

pytestmark = pytest.mark.gpu


def test_grown_chunks_in_another_process():
    rng = np.random.default_rng(19)
    c = Chunks(pic.GQA, pic.BF16, 2, 64, 64, [200, 200, 300], layers=2, capacity=64 * 16)
    c.append(rng, [130, 0, 7], layer=0)
    c.append(rng, [70, 5, 257], layer=1)
    c.append(rng, [0, 0, 64], layer=0)
    c.store.put(3, 100, *(L.draw(rng, pic.BF16, 2, 100, 2, 64) for _ in range(2)), L.stream())
    torch.cuda.synchronize()
    q = L.draw(rng, pic.BF16, 1, 4, 64)
    ids = [c.ids[0], 3, c.ids[1], c.ids[2]]
    ctx = mp.get_context("spawn")
    queue = ctx.Queue()
    child = ctx.Process(target=append_ipc_child.run, args=(c.store.export(), 2, 64, ids, q.float().cpu().numpy(), queue))
    child.start()
    try:
        res = queue.get(timeout=240)
    finally:
        child.join(timeout=60)
    assert "error" not in res, res.get("error")
    assert child.exitcode == 0
    # (chunk 1 holds nothing in layer 0: it is not handed over)
    assert res["lookup"] == {ids[0]: 70, 3: 100, ids[2]: pic.ERR_NOT_FOUND, ids[3]: 71}
    assert set(res["refused"].values()) == {pic.ERR_INVALID}, res["refused"]
    for layer in range(2):
        k, v = torch.zeros(100, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(100, 2, 64, dtype=torch.bfloat16, device="cuda")
        pic.debug_gather(c.store, [3], k, v, L.stream(), layer)
        torch.cuda.synchronize()
        want = [torch.cat([torch.cat(x[layer][0])[:70], y, torch.cat(x[layer][2])[:71]]) for x, y in ((c.k, k), (c.v, v))]
        for got, w in zip((res["k"][layer], res["v"][layer]), want):
            assert np.array_equal(got, w.float().cpu().numpy())
    ref, z = L.attend(q, *want, 0.125)
    L.check(pic.BF16, torch.from_numpy(res["out"]), torch.from_numpy(res["lse"]), ref, z)
