"""Child side of the 4-bit store's hand-over test (test_gpu_fp4.py): imports the parent's
store in a fresh process and links its chunk 9. Not collected by pytest (no test_ prefix)."""
import traceback


def run(blob, q_bits, results):
    try:
        import torch

        from paper_2602_01519_amd import pic

        torch.cuda.set_device(0)
        with pic.Store.import_(blob) as store:
            q = torch.from_numpy(q_bits).cuda()
            out = torch.empty_like(q)
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
            pic.link_attn(store, [0, 1], [9], [0, q.shape[0]], None, q.shape[1], q, None, None, 0.125, out, lse)
            torch.cuda.synchronize()
            results.put((out.cpu().numpy(), lse.cpu().numpy()))
    except Exception:
        results.put(traceback.format_exc())
        raise
