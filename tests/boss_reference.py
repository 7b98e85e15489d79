"""Plain fp64 restatement (NumPy) of the operators that train the Boss: instance-keyed dropout, the gradient of the instance loss, and
ragged attention with a relative position bias.  Test infrastructure; shares nothing with the CUDA library."""
import math

import numpy as np

U = np.uint64
MASK = U(0xFFFFFFFF)


def philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10: four arrays of output words from counters and keys that broadcast against each other."""
    c0, c1, c2, c3, k0, k1 = (a.copy() for a in np.broadcast_arrays(*(np.asarray(x, dtype=U) for x in (c0, c1, c2, c3, k0, k1))))
    with np.errstate(over="ignore"):
        for _ in range(10):
            p0, p1 = U(0xD2511F53) * c0, U(0xCD9E8D57) * c2
            c0, c1, c2, c3 = (p1 >> U(32)) ^ c1 ^ k0, p1 & MASK, (p0 >> U(32)) ^ c3 ^ k1, p0 & MASK
            k0, k1 = (k0 + U(0x9E3779B9)) & MASK, (k1 + U(0xBB67AE85)) & MASK
    return c0, c1, c2, c3


def _split(x):
    x = int(x) % 2**64
    return x & 0xFFFFFFFF, x >> 32


def instance_key(seed, step, ident):
    w = philox(*_split(ident), *_split(step), *_split(seed))
    return int(w[2]), int(w[3])


def draws(key, blocks, site):
    """Sixteen-bit draws of the blocks: [..., 8]."""
    blocks = np.asarray(blocks, dtype=U)
    w = philox(blocks & MASK, blocks >> U(32), site, 0, *key)
    out = np.empty(blocks.shape + (8,), dtype=np.int64)
    for i in range(4):
        out[..., 2 * i] = w[i] & U(0xFFFF)
        out[..., 2 * i + 1] = w[i] >> U(16)
    return out


def threshold(p):
    return min(65535, int(math.floor(65536.0 * float(np.float32(p)) + 0.5)))


def dropout_factor(rows, cols, p, seed, step, site, ident):
    """0 or the scale, for one instance of `rows` x `cols` elements."""
    t, groups = threshold(p), -(-cols // 8)
    block = np.arange(rows)[:, None] * groups + np.arange(groups)[None, :]
    kept = draws(instance_key(seed, step, ident), block, site).reshape(rows, groups * 8)[:, :cols] >= t
    return kept * (65536.0 / (65536 - t))


def attention_factor(heads, lq, lk, p, seed, step, site, ident):
    t, n = threshold(p), -(-lk // 32)
    h, i, j = np.arange(heads)[:, None, None], np.arange(lq)[None, :, None], np.arange(lk)[None, None, :]
    block = ((h * lq + i) * n + j // 32) * 4 + (j // 2) % 4
    half = np.broadcast_to(2 * ((j // 8) % 4) + j % 2, block.shape)
    u = np.take_along_axis(draws(instance_key(seed, step, ident), block, site), half[..., None], axis=-1)[..., 0]
    return (u >= t) * (65536.0 / (65536 - t))


def bucket(delta, buckets, distance, bidirectional):
    nb = buckets // 2 if bidirectional else buckets
    e = nb // 2
    n = abs(delta) if bidirectional else max(0, -delta)
    b = 0
    for k in range(nb):
        low = k if k < e else math.ceil(e * (distance / e) ** ((k - e) / (nb - e)) * (1 - 1e-9))
        if low <= n:
            b = k
    return b + (nb if bidirectional and delta > 0 else 0)


def row_losses(x, labels):
    top = x.max(axis=1)
    lse = top + np.log(np.exp(x - top[:, None]).sum(axis=1))
    return np.where(labels >= 0, lse - x[np.arange(len(x)), np.maximum(labels, 0)], 0.0)


def loss_grad(x, labels, factor):
    """Gradient of sum_r factor_r l_r."""
    e = np.exp(x - x.max(axis=1, keepdims=True))
    g = e / e.sum(axis=1, keepdims=True)
    g[np.arange(len(x)), np.maximum(labels, 0)] -= 1.0
    return g * np.where(labels >= 0, factor, 0.0)[:, None]


def attention_sequence(q, k, v, scale, causal, table=None, distance=0, bidirectional=True, factor=None, dout=None):
    """One sequence: q [lq, h, d], k / v [lk, hk, d].  Returns out, or a dict with the gradients and the sums of absolute terms that
    error bounds are stated in."""
    lq, h, d = q.shape
    lk, hk = k.shape[:2]
    rel = np.arange(lk)[None, :] - (np.arange(lq) + lk - lq)[:, None]
    if table is not None:
        span = range(int(rel.min(initial=0)), int(rel.max(initial=0)) + 1)
        of = np.array([bucket(x, table.shape[0], distance, bidirectional) for x in span])
        b = of[rel - span[0]] if rel.size else np.zeros(rel.shape, dtype=int)
    kk, vv = np.repeat(k, h // hk, axis=1), np.repeat(v, h // hk, axis=1)
    got = {n: np.zeros(s) for n, s in (("out", q.shape), ("out_abs", q.shape), ("dq", q.shape), ("dq_abs", q.shape), ("dk", k.shape), ("dk_abs", k.shape),
                                        ("dv", v.shape), ("dv_abs", v.shape))}
    if table is not None:
        got["dtable"], got["dtable_abs"] = np.zeros(table.shape), np.zeros(table.shape)
    for a in range(h):
        s = q[:, a] @ kk[:, a].T * scale
        if table is not None:
            s = s + table[b, a]
        if causal:
            s = np.where(rel > 0, -np.inf, s)
        top = s.max(axis=1, keepdims=True, initial=-np.inf)
        e = np.exp(s - np.where(np.isneginf(top), 0.0, top))
        total = e.sum(axis=1, keepdims=True)
        p = e / np.where(total == 0, 1.0, total)
        f = np.ones_like(p) if factor is None else factor[a]
        got["out"][:, a] = (p * f) @ vv[:, a]
        got["out_abs"][:, a] = (p * f) @ np.abs(vv[:, a])
        if dout is None:
            continue
        g = dout[:, a]
        dp = g @ vv[:, a].T * f
        D = (p * dp).sum(axis=1, keepdims=True)
        ds = p * (dp - D)
        ds_abs = p * (np.abs(g) @ np.abs(vv[:, a]).T * f + (p * np.abs(dp)).sum(axis=1, keepdims=True))
        got["dq"][:, a] = ds @ kk[:, a] * scale
        got["dq_abs"][:, a] = ds_abs @ np.abs(kk[:, a]) * scale
        c = a // (h // hk)
        got["dk"][:, c] += ds.T @ q[:, a] * scale
        got["dk_abs"][:, c] += ds_abs.T @ np.abs(q[:, a]) * scale
        got["dv"][:, c] += (p * f).T @ g
        got["dv_abs"][:, c] += (p * f).T @ np.abs(g)
        if table is not None:
            np.add.at(got["dtable"][:, a], b, ds)
            np.add.at(got["dtable_abs"][:, a], b, ds_abs)
    return got
