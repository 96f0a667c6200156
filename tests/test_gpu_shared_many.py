"""Shared links of more requests than a kernel argument names: own KV laid out by the call's tables."""
import numpy as np
import pytest

from test_gpu_shared import SHAPES, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,q_len", [("bf16-64", 1), ("bf16-64", 9), ("bf16-128", 1), ("bf16-128", 5), ("f32-40", 1), ("f32-64", 2), ("mla", 1),
                                        ("fp4-64", 1)])
def test_more_than_128_requests(name, q_len):
    shape = next(s for s in SHAPES if s[0] == name)
    rng = np.random.default_rng(q_len)
    per = [1, 100, 0, 60]
    b = Batch(rng, *shape[1:], per, [[70], [130, 20], [], [64]], [[5] if r % 7 == 0 else [] for r in range(161)], [q_len] * 161,
              own=[int(x) for x in rng.integers(0, 70, 161)])
    b.check(*b.call(), label="call")
    with b.plan() as plan:
        b.check(*b.run(plan), label="plan")
