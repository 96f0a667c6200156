"""Child side of test_gpu_append_import.py: imports a store with grown chunks, reads them back and links them.
Not collected by pytest (no test_ prefix)."""
import traceback


def run(blob, hkv, d, ids, q, out_q):
    try:
        import torch

        from paper_2602_01519_amd import pic

        torch.cuda.set_device(0)
        store = pic.Store.import_(blob)
        res = {"lookup": {}, "k": {}, "v": {}}
        for i in ids:
            try:
                res["lookup"][i] = store.lookup(i)
            except pic.PicError as e:
                res["lookup"][i] = e.status
        held = [i for i in ids if res["lookup"][i] > 0]
        n = sum(res["lookup"][i] for i in held)
        for layer in range(2):
            k, v = (torch.zeros(n, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            pic.debug_gather(store, held, k, v, layer=layer)
            torch.cuda.synchronize()
            res["k"][layer], res["v"][layer] = (x.float().cpu().numpy() for x in (k, v))
        qd = torch.from_numpy(q).to(torch.bfloat16).cuda()
        out = torch.zeros_like(qd)
        lse = torch.zeros(qd.shape[:2], dtype=torch.float32, device="cuda")
        pic.link_decode(store, [0, len(held)], held, [0, 1], None, qd.shape[1], qd, None, None, 0.125, out, lse, layer=1)
        torch.cuda.synchronize()
        res["out"], res["lse"] = out.float().cpu().numpy(), lse.cpu().numpy()
        refused = {"open": lambda: store.open(9, 5), "append": lambda: store.append(held[:1], [0, 1], qd[:, :hkv], qd[:, :hkv]),
                   "truncate": lambda: store.truncate(held[:1], [1])}
        res["refused"] = {}
        for name, call in refused.items():
            try:
                call()
                res["refused"][name] = 0
            except pic.PicError as e:
                res["refused"][name] = e.status
        store.close()
        out_q.put(res)
    except Exception:
        out_q.put({"error": traceback.format_exc()})
        raise
