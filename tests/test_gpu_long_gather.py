"""Read-back of lists of more than 2^30 tokens, and the refusal of those past 2^31 - 1."""
import pytest
import torch

import link_model as L
from paper_2602_01519_amd import pic

pytestmark = pytest.mark.gpu


def test_lists_past_a_billion_tokens():
    n = 1 << 20
    with pic.Store(pic.MLA, pic.BF16, 1, 8, 8, 2 * n) as store:
        k = torch.randn(n, 1, 8, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
        k2 = -k[:n - 3]
        store.put(1, n, k, None, L.stream())
        store.put(2, n - 3, k2, None, L.stream())
        for ids in ([1] * 1025, [1] * 700 + [2] + [1] * 700):
            total = sum(n if i == 1 else n - 3 for i in ids)
            assert total > 1 << 30
            out = torch.empty(total, 1, 8, dtype=torch.bfloat16, device="cuda")
            pic.debug_gather(store, ids, out, None, L.stream())
            torch.cuda.synchronize()
            at = 0
            for i in ids:
                want = k if i == 1 else k2
                assert torch.equal(out[at:at + len(want)], want), at
                at += len(want)
            del out
        small = torch.full((64, 1, 8), 5.0, dtype=torch.bfloat16, device="cuda")
        with pytest.raises(pic.PicError) as e:        # (refused on the host: nothing is written)
            pic.debug_gather(store, [1] * 2048, small, None, L.stream())
        assert e.value.status == pic.ERR_INVALID
        torch.cuda.synchronize()
        assert bool((small == 5).all())
