"""Selected blocks where the heads of a kv head take several workgroups (over 4 heads in fp32, over 16 in
bf16): a unit's blocks are shared out only as far as all of these leave CUs free."""
import copy

import numpy as np
import pytest
import torch

import link_model as L
from paper_2602_01519_amd import pic
from test_gpu_sparse import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,group,columns", [(pic.F32, 64, 8, 2), (pic.F32, 128, 5, 2), (pic.F32, 64, 12, 3),
                                                   (pic.BF16, 128, 20, 2), (pic.BF16, 64, 40, 3)])
@pytest.mark.parametrize("full", [True, False])
def test_units_of_several_workgroups(dtype, d, group, columns, full):
    """A batch whose units fill half of the CUs, its workgroups all of them: the result has the bits of
    captured calls, which never share a unit out. A smaller batch is shared out: other sums, other bits."""
    rng = np.random.default_rng(group)
    cus, n = torch.cuda.get_device_properties(0).multi_processor_count, 8
    batch = cus // 4 if full else cus // (8 * columns)
    c = Case(rng, dtype, 2, d, group, [700, 900, 330, 1000], [[i % 4] for i in range(batch)], [1] * batch, own=[7] * batch)
    got = c.call(n, 1, 1)
    c.check(got, n, 1, 1)
    parts = []
    for at in range(0, batch, 32):             # (a capture takes up to 32 query tokens)
        m = min(32, batch - at)
        p = copy.copy(c)
        p.links, p.starts, p.q_len, p.own = c.links[at:at + m], c.starts[at:at + m], [1] * m, [8] * m
        p.q, p.ko, p.vo = c.q[at:at + m], c.ko[8 * at:8 * (at + m)], c.vo[8 * at:8 * (at + m)]
        bufs, g = p.buffers(n), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            p.call(n, 1, 1, bufs=bufs)
        for _ in range(2):
            g.replay()
        p.check(bufs, n, 1, 1)
        parts.append(bufs)
    out, lse, blocks = (torch.cat(x) for x in zip(*parts))
    same = [torch.equal(a, b) for a, b in zip((out, lse, blocks), got)]
    assert same[2] and (same[0] and same[1]) == full
