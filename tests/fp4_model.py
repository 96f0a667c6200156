"""The 4-bit cache and link attention over it in 64 bits on the host, written from the
definition in include/pic.h (numpy, no code of the library). Not collected by pytest.

Tolerances. Cached keys and values and the queries are exact in the matrix products; what
the kernels round is each probability once to bf16 (at most 2^-8 of it) and each output
once (2^-8 of it), so per element

    |out - ref| <= 2^-8 |ref| + 2^-8 W + slack,   W = sum_j softmax_j |v_j|

(the sum of probabilities is taken before they are rounded). Scores are sums of D products
in fp32, off by at most D 2^-24 sum|q k| scale; a relative change e of every probability moves
out by at most 2 e W, and lse by e. Sums of n probabilities in fp32 (partial sums of lanes
and pieces: fewer than n steps) add n 2^-24. exp2, the scale and the log-sum-exp's own
rounding add a few 2^-24 of the logit's size. What is smaller than 2^-126 may be flushed to
zero: each of n probabilities, whose sum is at least 1/2 (the largest is about 1 in its own
unit), and the output: at most (n + 1) 2^-126 (1 + max|v|) in all."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
BORDER = [(0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True),
          (5.0, False)]           # (border above code i, whether a value on it goes up)


def bf16(x):
    """fp32 / fp64 array rounded to bf16 (nearest even), as float64; NaN and infinities kept."""
    u = np.asarray(x, np.float32).view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32)
    r = np.where(np.isfinite(np.asarray(x, np.float32)), r, u)
    return r.view(np.float32).astype(np.float64)


def bits(x):
    """bf16 bit patterns (int16) of bf16-valued float64."""
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16).view(np.int16)


def stored(x):
    """The numbers a 4-bit store keeps for rows x [..., d] (bf16-valued float64)."""
    b = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    a = np.abs(b).max(-1)                      # NaN where the block has one
    e = np.full(a.shape, -126)
    for k in range(-126, 126):                 # the smallest exponent with a < 7 * 2^k, 125 at most
        e = np.where((e == k) & ~(a < 7 * 2.0 ** k) & (k < 125), k + 1, e)
    scale = 2.0 ** e[..., None].astype(np.float64)
    y = np.abs(b) / scale
    code = sum(((y >= t) if up else (y > t)).astype(int) for t, up in BORDER)
    out = np.copysign(GRID[code] * scale, b)
    out[np.isnan(a)] = np.nan
    return out.reshape(x.shape)


def attend(q, k, v, scale, seen):
    """Rows q [lq][hq][d] over keys k, v [n][hkv][d]; seen [lq][n]. (out, lse, tolerance of out, of lse)."""
    lq, hq, d = q.shape
    hkv, n = k.shape[1], k.shape[0]
    g = hq // hkv
    out, lse = np.zeros(q.shape), np.full((lq, hq), -np.inf)
    tol, tl = np.zeros(q.shape), np.zeros((lq, hq))
    u = 2.0 ** -24
    some = seen.any(1)
    for h in range(hq):
        kh, vh = k[:, h // g], v[:, h // g]
        s = np.where(seen, scale * (q[:, h] @ kh.T), -np.inf)[some]
        if not len(s):
            continue
        size = np.where(seen, scale * (np.abs(q[:, h]) @ np.abs(kh).T), 0.0)[some].max(1)
        m = s.max(1)
        p = np.exp(s - m[:, None])
        total = p.sum(1)
        w = p / total[:, None]
        o, z = w @ vh, m + np.log(total)
        logit = np.where(np.isfinite(s), np.abs(s), 0.0).max(1)
        e = u * (d * size + 4 * logit + n + 16)
        tl[some, h] = e + u * 4 * np.abs(z)
        tol[some, h] = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 4 * e[:, None]) * (w @ np.abs(vh)) + \
            (n + 1) * 2.0 ** -126 * (1 + np.abs(vh).max())
        out[some, h], lse[some, h] = o, z
    return out, lse, tol, tl


def batch(q, chunks, links, starts, k_own, v_own, q_off, own_off, scale, limits=None):
    """Every request of a batch; chunks: id -> (k, v) stored values."""
    res = [[], [], [], []]
    for r, ids in enumerate(links):
        q0, q1 = q_off[r], q_off[r + 1]
        lq = q1 - q0
        ks = [chunks[c][0][s:] for c, s in zip(ids, starts[r])]
        vs = [chunks[c][1][s:] for c, s in zip(ids, starts[r])]
        doc = sum(x.shape[0] for x in ks)
        ls = 0
        if own_off is not None:
            ls = own_off[r + 1] - own_off[r]
            ks.append(k_own[own_off[r]:own_off[r + 1]])
            vs.append(v_own[own_off[r]:own_off[r + 1]])
        hkv, d = next(iter(chunks.values()))[0].shape[1:]
        k = np.concatenate(ks) if ks else np.zeros((0, hkv, d))
        v = np.concatenate(vs) if vs else np.zeros((0, hkv, d))
        seen = np.zeros((lq, doc + ls), bool)
        for i in range(lq):
            seen[i, :doc if limits is None else limits[q0 + i]] = True
            seen[i, doc:doc + max(0, i + 1 + ls - lq)] = True
        for a, b in zip(res, attend(q[q0:q1], k, v, scale, seen)):
            a.append(b)
    return [np.concatenate(a) for a in res]
