"""Value widths past those of the generic kernel are refused, not left unwritten."""
import pytest
import torch

from paper_2602_01519_amd import pic

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [pic.F32, pic.BF16])
@pytest.mark.parametrize("d_v,ok", [(512, True), (520, False), (768, False)])
def test_values_wider_than_the_kernel(dtype, d_v, ok):
    t = torch.float32 if dtype == pic.F32 else torch.bfloat16
    with pic.Store(pic.GQA, dtype, 1, 64, d_v, 128) as store:
        store.put(1, 70, torch.zeros(70, 1, 64, dtype=t, device="cuda"), torch.ones(70, 1, d_v, dtype=t, device="cuda"))
        out = torch.full((3, 2, d_v), 7.0, dtype=t, device="cuda")
        for call in (pic.link_attn, pic.link_decode):
            out.fill_(7.0)
            args = (store, [0, 1], [1], [0, 3], None, 2, torch.zeros(3, 2, 64, dtype=t, device="cuda"), None, None, 1.0, out)
            if ok:
                call(*args)
            else:
                with pytest.raises(pic.PicError) as e:
                    call(*args)
                assert e.value.status == pic.ERR_UNSUPPORTED
            torch.cuda.synchronize()
            assert bool((out == (1.0 if ok else 7.0)).all())
