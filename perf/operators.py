"""The Boss's training operators, as measured cases: dropout keyed by instance, the gradient of the instance loss, and attention
over ragged sentences with a learned relative position bias.

``run`` computes each operator in its plain form (elementary torch operations in 32 bits, rounded once at the end) or, where
``own`` is true, by the calls of ``paper_1905_03381_b200.binding``.  ``exact`` restates the definitions in 64 bits.

The draws of a dropout are part of its definition: Philox4x32-10, keyed per instance by (seed, instance id, step), counted per block
of eight elements; sixteen bits decide one element.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SEED = 20190503   # seed of the Philox draws; the step number comes from the inputs' seed


# ---------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one short sentence's activations: the smallest call, where launch latency is all there is
        {"name": "dropout_one_sentence", "op": "dropout", "dtype": "bf16", "sentences": 1, "len_lo": 17, "len_hi": 17, "cols": 512,
         "p": 0.1, "residual": True},
        # one residual connection of a translation batch of about 25,000 target tokens
        {"name": "dropout_translation_tokens", "op": "dropout", "dtype": "bf16", "sentences": 368, "len_lo": 8, "len_hi": 128, "cols": 512,
         "p": 0.1, "residual": True},
        # fp32 classifier activations of an image batch, one row an instance, odd width, the backward direction (no residual)
        {"name": "dropout_image_rows_odd", "op": "dropout", "dtype": "f32", "sentences": 0, "rows": 30011, "cols": 1001,
         "p": 0.5, "residual": False},
        # the tiny reference's logits: 4,096 rows of 10 classes
        {"name": "loss_grad_tiny", "op": "loss", "dtype": "f32", "sentences": 0, "rows": 4096, "cols": 10, "weights": False},
        # the image benchmark's logits over a batch of accepted instances, weighted by 1 / acceptance probability
        {"name": "loss_grad_image", "op": "loss", "dtype": "f32", "sentences": 0, "rows": 39000, "cols": 100, "weights": True},
        # the translation benchmark's logits: about 25,000 token rows over 32,000 words, summed per sentence
        {"name": "loss_grad_translation", "op": "loss", "dtype": "bf16", "sentences": 368, "len_lo": 8, "len_hi": 128, "cols": 32000,
         "weights": True},
        # the widest vocabulary of the loss sweep, one word short of it: rows that start at every alignment
        {"name": "loss_grad_wide_odd", "op": "loss", "dtype": "bf16", "sentences": 0, "rows": 4096, "cols": 131071, "weights": False},
        # one new token over a long context, the serving direction
        {"name": "attention_one_token", "op": "attention", "dtype": "bf16", "sentences": 4, "len_lo": 4001, "len_hi": 4001, "q_len": 1,
         "heads": 16, "kv_heads": 4, "dim": 128, "causal": True, "buckets": 32, "distance": 128, "p": 0.0, "train": False},
        # self-attention of a translation batch, forward only (validation)
        {"name": "attention_translation_eval", "op": "attention", "dtype": "bf16", "sentences": 368, "len_lo": 8, "len_hi": 128, "q_len": 0,
         "heads": 8, "kv_heads": 8, "dim": 64, "causal": False, "buckets": 32, "distance": 128, "p": 0.0, "train": False},
        # the same in training: dropout on the probabilities, forward and every gradient
        {"name": "attention_translation_train", "op": "attention", "dtype": "bf16", "sentences": 368, "len_lo": 8, "len_hi": 128, "q_len": 0,
         "heads": 8, "kv_heads": 8, "dim": 64, "causal": True, "buckets": 32, "distance": 128, "p": 0.1, "train": True},
        # long documents, shared key heads, both directions
        {"name": "attention_long_train", "op": "attention", "dtype": "bf16", "sentences": 2, "len_lo": 4096, "len_hi": 4096, "q_len": 0,
         "heads": 16, "kv_heads": 4, "dim": 128, "causal": True, "buckets": 32, "distance": 128, "p": 0.0, "train": True},
        # fp32, an odd head width, sentences of one token to a few hundred
        {"name": "attention_f32_odd_train", "op": "attention", "dtype": "f32", "sentences": 24, "len_lo": 1, "len_hi": 301, "q_len": 0,
         "heads": 5, "kv_heads": 5, "dim": 40, "causal": False, "buckets": 20, "distance": 50, "p": 0.2, "train": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["dropout", "loss", "attention", "attention"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    ragged = rng.random() < 0.6
    if op == "dropout":
        cols = _log_int(rng, 64, 4099)
        rows = _log_int(rng, 16, max(17, 40_000_000 // cols))
        case = {"op": op, "dtype": dtype, "cols": cols, "p": rng.choice([0.1, 0.2, 0.5]), "residual": rng.random() < 0.5}
    elif op == "loss":
        cols = _log_int(rng, 10, 131072)
        rows = _log_int(rng, 16, max(17, min(65536, (260_000_000 if dtype == "f32" else 520_000_000) // cols)))
        case = {"op": op, "dtype": dtype, "cols": cols, "weights": rng.random() < 0.5}
    else:
        causal, train = rng.random() < 0.5, rng.random() < 0.6
        dim = rng.choice([32, 64, 64, 96, 128]) if dtype == "bf16" else rng.choice([24, 40, 64])
        kv = rng.choice([1, 2, 4])
        heads = kv * rng.choice([1, 2, 4])
        one = rng.random() < 0.25
        hi = _log_int(rng, 1, 32768 if one else 4096 if dtype == "bf16" else 512)
        lo = max(1, int(hi * rng.choice([0.1, 0.5, 1.0])))
        # pairs x heads x dim stay below the largest listed case; one-token queries are held to a few hundred megabytes of keys
        room = 1.5e8 / (float(hi) * heads * dim) if one else (1.2e10 if dtype == "bf16" else 1.0e9) / (float(hi) * hi * heads * dim)
        sentences = max(1, min(_log_int(rng, 1, 512), int(room)))
        distance = rng.choice([64, 128, 200])
        return {"op": op, "dtype": dtype, "sentences": sentences, "len_lo": lo, "len_hi": hi, "q_len": 1 if one else 0, "heads": heads,
                "kv_heads": kv, "dim": dim, "causal": causal, "buckets": rng.choice([16, 32, 64]), "distance": distance,
                "p": rng.choice([0.0, 0.1]), "train": train and not one, "lens_seed": rng.randrange(1 << 30)}
    if ragged:
        hi = max(1, min(rows, rng.choice([16, 60, 128, 500])))
        lo = max(1, hi // rng.choice([1, 4, 16]))
        case.update(sentences=max(1, rows * 2 // (lo + hi)), len_lo=lo, len_hi=hi, lens_seed=rng.randrange(1 << 30))
    else:
        case.update(sentences=0, rows=rows)
    return case


def _lengths(case):
    r = random.Random(case.get("lens_seed", 5))
    return [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["sentences"])]


def _pairs(case):
    """(query rows, key rows, scored (query, key) pairs of one head)."""
    q_rows = k_rows = pairs = 0
    for k in _lengths(case):
        q = case["q_len"] or k
        q_rows, k_rows = q_rows + q, k_rows + k
        pairs += sum(max(0, i + k - q + 1) for i in range(q)) if case["causal"] else q * k
    return q_rows, k_rows, pairs


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "attention":
        q_rows, k_rows, pairs = _pairs(case)
        q, kv = q_rows * case["heads"] * case["dim"] * es, k_rows * case["kv_heads"] * case["dim"] * es
        if case["train"]:   # forward: q, k, v -> o; backward: q, k, v, do -> dq, dk, dv
            return {"bytes": 5 * q + 6 * kv, "flops": 14.0 * case["dim"] * pairs * case["heads"]}
        return {"bytes": 2 * q + 2 * kv, "flops": 4.0 * case["dim"] * pairs * case["heads"]}
    rows = sum(_lengths(case)) if case["sentences"] else case["rows"]
    n = rows * case["cols"]
    if case["op"] == "dropout":
        return {"bytes": n * es * (3 if case["residual"] else 2) + rows * 4, "flops": 2.0 * n}
    return {"bytes": 2 * n * es + rows * 8, "flops": 5.0 * n}


# --------------------------------------------------------------------------------------------------------------- inputs

def _offsets(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(np.asarray(lens, dtype=np.int64))]).astype(np.int32), device=DEV)


def _draw_inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(shape, std=1.0, t=dtype):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(t)

    s = {"case": case, "step": seed}
    lens = _lengths(case) if case["sentences"] else None
    if case["op"] == "attention":
        q_lens = [case["q_len"] or k for k in lens]
        s["k_off"] = _offsets(lens)
        s["q_off"] = _offsets(q_lens) if case["q_len"] else s["k_off"]
        s["max_q"], s["max_k"] = max(q_lens), max(lens)
        nq, nk, h, kv, d = sum(q_lens), sum(lens), case["heads"], case["kv_heads"], case["dim"]
        s["q"], s["k"], s["v"] = normal((nq, h, d)), normal((nk, kv, d)), normal((nk, kv, d))
        s["table"] = normal((case["buckets"], h), 0.5, torch.float32)
        if case["train"]:
            s["dout"] = normal((nq, h, d))
        instances = len(lens)
    else:
        rows = sum(lens) if lens else case["rows"]
        instances = len(lens) if lens else rows
        s["off"] = _offsets(lens) if lens else None
        if case["op"] == "dropout":
            s["x"] = normal((rows, case["cols"]))
            s["res"] = normal((rows, case["cols"])) if case["residual"] else None
        else:
            s["x"] = normal((rows, case["cols"]), 3.0)
            s["labels"] = torch.randint(0, case["cols"], (rows,), generator=g, device=DEV, dtype=torch.int32)
            s["labels"][torch.rand(rows, generator=g, device=DEV) < 0.01] = -1   # padding rows
            s["w"] = 1.0 / (0.1 + 0.9 * torch.rand(instances, generator=g, device=DEV)) if case["weights"] else None
    # the batch list: ascending stored rows of a pool about twice the batch
    s["row_idx"] = (2 * torch.arange(instances, device=DEV) + torch.randint(0, 2, (instances,), generator=g, device=DEV)).to(torch.int32)
    return s


def prepare(case, seed):
    s = _draw_inputs(case, seed)
    if own:
        from paper_1905_03381_b200 import binding as B
        x = s["q"] if case["op"] == "attention" else s["x"]
        s["aa"] = B.AutoAssist(max_rows=x.shape[0], max_d=max(16, case.get("dim", 16)), device="cuda:0")
        if case["op"] == "attention":
            s["attn"] = B.attention(s["q"], s["k"], s["v"], s["q_off"], s["k_off"], s["max_q"], s["max_k"], causal=case["causal"])
            s["bias"] = B.rel_bias(s["table"], case["distance"], bidirectional=not case["causal"])
            s["drop"] = B.dropout_rule(case["p"], SEED, s["step"], site=3, row_idx=s["row_idx"]) if case["p"] else None
            s["out"] = torch.empty_like(s["q"])
            if case["train"]:
                s["dq"], s["dk"], s["dv"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
                s["dtable"] = torch.empty_like(s["table"])
                s["scratch"] = s["aa"].rel_attention_scratch(s["attn"], s["bias"])
        elif case["op"] == "dropout":
            s["rule"] = B.dropout_rule(case["p"], SEED, s["step"], site=1, row_idx=s["row_idx"])
            s["out"] = torch.empty_like(s["x"])
        else:
            s["logits"] = B.logits_desc(s["x"])
            s["grad"], s["loss"] = torch.empty_like(s["x"]), torch.empty(s["row_idx"].numel(), device=DEV)
    return s


# ----------------------------------------------------------------------------------------------------------- one pass

def run(state):
    s, case = state, state["case"]
    if own:
        return _run_own(s, case)
    if case["op"] == "attention":
        return _plain_attention(s, case)
    return _plain_dropout(s, case) if case["op"] == "dropout" else _plain_loss(s, case)


def _run_own(s, case):
    aa = s["aa"]
    if case["op"] == "dropout":
        aa.aa_dropout(s["x"], s["rule"], s["out"], residual=s["res"], offsets=s["off"])
        return s["out"]
    if case["op"] == "loss":
        aa.aa_instance_loss_grad(s["logits"], s["labels"], s["grad"], offsets=s["off"], weight=s["w"], mean=True, out_loss=s["loss"])
        return {"grad": s["grad"], "loss": s["loss"]}
    aa.aa_rel_attention(s["attn"], s["out"], bias=s["bias"], dropout=s["drop"])
    if not case["train"]:
        return s["out"]
    aa.aa_rel_attention_grad(s["attn"], s["dout"], s["dq"], s["dk"], s["dv"], s["scratch"], bias=s["bias"], dropout=s["drop"], dtable=s["dtable"])
    return {"out": s["out"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"], "dtable": s["dtable"]}


# --------------------------------------------------------------------------------------------------------- plain forms

_M32 = 0xFFFFFFFF


def _mul32(a, c):
    """High and low words of the 64-bit product of 32-bit words held in int64."""
    t, u = c * (a & 0xFFFF), c * (a >> 16)
    return (u + (t >> 16)) >> 16, ((u << 16) + t) & _M32


def _philox(c0, c1, c2, c3, k0, k1):
    for _ in range(10):
        h0, l0 = _mul32(c0, 0xD2511F53)
        h1, l1 = _mul32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return c0, c1, c2, c3


def _instance_keys(row_idx, step):
    z = torch.zeros_like(row_idx, dtype=torch.int64)
    return _philox(row_idx.long(), z, z + (step & _M32), z + (step >> 32), z + (SEED & _M32), z + (SEED >> 32))[2:]


def _halves(block, k0, k1, site):
    """Eight 16-bit draws of each block: the last dimension of the answer."""
    z = torch.zeros_like(block)
    w = _philox(block & _M32, block >> 32, z + site, z, k0 + z, k1 + z)
    return torch.stack([w[0] & 0xFFFF, w[0] >> 16, w[1] & 0xFFFF, w[1] >> 16, w[2] & 0xFFFF, w[2] >> 16, w[3] & 0xFFFF, w[3] >> 16], -1)


def _threshold(p):
    return min(65535, int(math.floor(65536.0 * p + 0.5)))


def _segment_of_rows(off, rows):
    return torch.bucketize(torch.arange(rows, device=DEV, dtype=torch.int32), off[1:], right=True)


def _plain_dropout(s, case):
    x, off, t = s["x"], s["off"], _threshold(case["p"])
    rows, cols = x.shape
    r = torch.arange(rows, device=DEV)
    seg = _segment_of_rows(off, rows) if off is not None else r
    a = r - off.long()[seg] if off is not None else torch.zeros_like(r)
    k0, k1 = (k[seg][:, None] for k in _instance_keys(s["row_idx"], s["step"]))
    groups = (cols + 7) // 8
    block = a[:, None] * groups + torch.arange(groups, device=DEV)[None, :]
    keep = _halves(block, k0, k1, 1).reshape(rows, groups * 8)[:, :cols] >= t
    y = torch.where(keep, x.float() * (65536.0 / (65536 - t)), torch.zeros((), device=DEV))
    if s["res"] is not None:
        y = y + s["res"].float()
    return y.to(x.dtype)


def _plain_loss(s, case):
    x, off, y = s["x"].float(), s["off"], s["labels"].long()
    rows = x.shape[0]
    n = s["row_idx"].numel()
    seg = _segment_of_rows(off, rows) if off is not None else torch.arange(rows, device=DEV)
    live = y >= 0
    top = x.max(dim=1, keepdim=True).values
    e = torch.exp(x - top)
    total = e.sum(dim=1, keepdim=True)
    at = y.clamp(min=0)[:, None]
    row_loss = torch.where(live, (top + torch.log(total) - x.gather(1, at))[:, 0], torch.zeros((), device=DEV))
    w = (s["w"] if s["w"] is not None else torch.ones(n, device=DEV)) / n
    factor = torch.where(live, w[seg], torch.zeros((), device=DEV))[:, None]
    grad = e / total
    grad.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
    grad = grad * factor
    loss = row_loss if off is None else torch.zeros(n, device=DEV).index_add_(0, seg, row_loss)
    return {"grad": grad.to(s["x"].dtype), "loss": loss}


def _lower_bounds(nb, distance):
    e = nb // 2
    return [k if k < e else int(math.ceil(e * (distance / e) ** ((k - e) / (nb - e)) * (1 - 1e-9))) for k in range(nb)]


def _buckets(delta, case):
    both = not case["causal"]
    nb = case["buckets"] // 2 if both else case["buckets"]
    lower = torch.tensor(_lower_bounds(nb, case["distance"]), device=DEV)
    n = delta.abs() if both else (-delta).clamp(min=0)
    b = torch.bucketize(n, lower, right=True) - 1
    return b + nb * (delta > 0) if both else b


def _padded(x, off, longest):
    """Rows of ragged sequences as [sequence, head, position, ...] with zeros behind each sequence's end, and what is real."""
    at = off[:-1].long()[:, None] + torch.arange(longest, device=DEV)[None, :]
    real = at < off[1:].long()[:, None]
    y = x[at.clamp(max=x.shape[0] - 1)].float() * real[:, :, None, None]
    return y.transpose(1, 2), real


def _plain_attention(s, case):
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    scale = 1.0 / math.sqrt(d)
    q, q_real = _padded(s["q"], s["q_off"], s["max_q"])
    k, k_real = _padded(s["k"], s["k_off"], s["max_k"])
    v, _ = _padded(s["v"], s["k_off"], s["max_k"])
    k, v = k.repeat_interleave(h // kv, 1), v.repeat_interleave(h // kv, 1)
    lq, lk = (s["q_off"][1:] - s["q_off"][:-1]).long(), (s["k_off"][1:] - s["k_off"][:-1]).long()
    i, j = torch.arange(s["max_q"], device=DEV), torch.arange(s["max_k"], device=DEV)
    delta = j[None, None, :] - i[None, :, None] - (lk - lq)[:, None, None]
    seen = q_real[:, :, None] & k_real[:, None, :]
    if case["causal"]:
        seen = seen & (delta <= 0)
    seen = seen[:, None]
    low = torch.full((), -math.inf, device=DEV)
    sc = q @ k.transpose(2, 3) * scale + s["table"][_buckets(delta, case)].permute(0, 3, 1, 2)
    sc = torch.where(seen, sc, low)
    top = sc.max(dim=3, keepdim=True).values
    top = torch.where(top == low, torch.zeros((), device=DEV), top)
    e = torch.exp(sc - top)
    total = e.sum(dim=3, keepdim=True)
    prob = e / torch.where(total == 0, torch.ones((), device=DEV), total)
    t = _threshold(case["p"])
    if t:
        n = (lk + 31) // 32
        head = torch.arange(h, device=DEV)
        row = (head[None, :, None] * lq[:, None, None] + i[None, None, :]) * n[:, None, None]
        chunks = (s["max_k"] + 31) // 32
        block = (row[..., None, None] + torch.arange(chunks, device=DEV)[:, None]) * 4 + torch.arange(4, device=DEV)[None, :]
        k0, k1 = (x[:, None, None, None, None] for x in _instance_keys(s["row_idx"], s["step"]))
        u = _halves(block, k0, k1, 3)                                         # [..., chunk, call, half]
        u = u.reshape(*u.shape[:-1], 4, 2).transpose(-3, -2)                  # key = 32 chunk + 8 (half // 2) + 2 call + half % 2
        keep = (u.reshape(*u.shape[:3], chunks * 32)[..., :s["max_k"]] >= t).float() * (65536.0 / (65536 - t))
    else:
        keep = None
    dropped = prob if keep is None else prob * keep
    q_at = q_real.nonzero(as_tuple=True)
    k_at = k_real.nonzero(as_tuple=True)

    def rows(x, at):
        return x.transpose(1, 2)[at]

    out = rows(dropped @ v, q_at).to(s["q"].dtype)
    if not case["train"]:
        return out
    do, _ = _padded(s["dout"], s["q_off"], s["max_q"])
    dv = dropped.transpose(2, 3) @ do
    dp = do @ v.transpose(2, 3)
    dp = dp if keep is None else dp * keep
    ds = prob * (dp - (prob * dp).sum(dim=3, keepdim=True))
    dq = ds @ k * scale
    dk = ds.transpose(2, 3) @ q * scale
    # the table's gradient: sums along the diagonals (rows reversed, padded by one row length, read one element short per row), then by bucket
    n_seq, _, r, c = ds.shape
    skew = torch.nn.functional.pad(ds.flip(2), (0, r)).reshape(n_seq, h, r * (r + c))[:, :, :r * (r + c - 1)]
    diagonal = skew.reshape(n_seq, h, r, r + c - 1).sum(dim=2)
    where = torch.arange(r + c - 1, device=DEV)[None, :] - (r - 1) - (lk - lq)[:, None]
    dtable = torch.zeros((case["buckets"], h), device=DEV).index_add_(0, _buckets(where, case).reshape(-1), diagonal.transpose(1, 2).reshape(-1, h))
    shared = (n_seq, kv, h // kv, c, d)
    dk, dv = dk.reshape(shared).sum(2), dv.reshape(shared).sum(2)
    return {"out": out, "dq": rows(dq, q_at).to(out.dtype), "dk": rows(dk, k_at).to(out.dtype), "dv": rows(dv, k_at).to(out.dtype),
            "dtable": dtable}


# ------------------------------------------------------------------------------------------------------- in 64 bits

def _draws64(key_of, block, site):
    """Sixteen-bit draws of the blocks (a numpy array of uint64) under one instance's key: [..., 8]."""
    def words(ctr, key):
        c, k = [np.array(x, dtype=np.uint64) for x in ctr], list(key)
        mask, m = np.uint64(0xFFFFFFFF), (np.uint64(0xD2511F53), np.uint64(0xCD9E8D57))
        for _ in range(10):
            a, b = m[0] * c[0], m[1] * c[2]
            c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & mask, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & mask]
            k = [(k[0] + 0x9E3779B9) % 2**32, (k[1] + 0xBB67AE85) % 2**32]
        return c

    ident, step = key_of
    key = [int(x) for x in words([ident % 2**32, ident >> 32, step % 2**32, step >> 32], [SEED % 2**32, SEED >> 32])[2:]]
    zero = np.zeros_like(block)
    w = np.stack(words([block & np.uint64(0xFFFFFFFF), block >> np.uint64(32), zero + np.uint64(site), zero], key), -1)
    return w.astype("<u4").view("<u2").reshape(*block.shape, 8)


def exact(case, seed):
    if case["op"] == "attention" and _pairs(case)[2] * case["heads"] > (1.0e8 if case["p"] else 6e8):
        return None
    s = _draw_inputs(case, seed)
    ids, step = s["row_idx"].cpu().tolist(), s["step"]
    if case["op"] == "attention":
        return _exact_attention(s, case, ids, step)
    off = s["off"].cpu().tolist() if s["off"] is not None else list(range(s["x"].shape[0] + 1))
    x = s["x"].double()
    cols = x.shape[1]
    if case["op"] == "dropout":
        t, groups = _threshold(case["p"]), -(-cols // 8)
        keep = np.empty((x.shape[0], cols), dtype=bool)
        if s["off"] is None and x.shape[0] > 100_000:
            return None
        for n, ident in enumerate(ids):
            a, b = off[n], off[n + 1]
            block = np.arange((b - a) * groups, dtype=np.uint64).reshape(b - a, groups)
            keep[a:b] = (_draws64((ident, step), block, 1).reshape(b - a, groups * 8) >= t)[:, :cols]
        y = x * torch.from_numpy(keep).to(DEV) * 65536.0 / (65536 - t)
        return y if s["res"] is None else y + s["res"].double()
    n = len(ids)
    grad, loss = torch.zeros_like(x), torch.zeros(n, dtype=torch.float64, device=DEV)
    span = torch.tensor(np.diff(np.asarray(off)), device=DEV)
    inst = torch.repeat_interleave(torch.arange(n, device=DEV), span)
    weight = torch.full((n,), 1.0 / n, dtype=torch.float64, device=DEV) if s["w"] is None else s["w"].double() / n
    label = s["labels"].long()
    picked = torch.nonzero(label >= 0)[:, 0]
    for at in picked.split(max(1, 400_000_000 // cols)):
        logp = torch.log_softmax(x[at], dim=1)
        one = label[at][:, None]
        loss.index_add_(0, inst[at], -logp.gather(1, one)[:, 0])
        g = logp.exp()
        g.scatter_add_(1, one, torch.full((at.numel(), 1), -1.0, dtype=torch.float64, device=DEV))
        grad[at] = g * weight[inst[at]][:, None]
    return {"grad": grad, "loss": loss}


def _exact_attention(s, case, ids, step):
    h, group, d = case["heads"], case["heads"] // case["kv_heads"], case["dim"]
    q, k, v, table = (s[n].double().requires_grad_(case["train"]) for n in ("q", "k", "v", "table"))
    qo, ko, t = s["q_off"].cpu().tolist(), s["k_off"].cpu().tolist(), _threshold(case["p"])
    both = not case["causal"]
    nb = case["buckets"] // 2 if both else case["buckets"]
    half = nb // 2
    of = np.zeros(max(s["max_k"], s["max_q"]) + 1, dtype=np.int64)      # bucket of each distance, counted up by the boundaries passed
    for b in range(1, nb):
        of[(b if b < half else math.ceil(half * math.exp(math.log(case["distance"] / half) * (b - half) / (nb - half)) * (1 - 1e-9))):] += 1
    of = torch.tensor(of, device=DEV)
    out = torch.zeros_like(q)
    grads = [torch.zeros_like(x) for x in (q, k, v, table)] if case["train"] else None
    for n, ident in enumerate(ids):
        lq, lk = qo[n + 1] - qo[n], ko[n + 1] - ko[n]
        qs, ks = slice(qo[n], qo[n + 1]), slice(ko[n], ko[n + 1])
        rel = torch.arange(lk, device=DEV)[None, :] - (torch.arange(lq, device=DEV) + lk - lq)[:, None]
        bucket = of[rel.abs()] + nb * (rel > 0) if both else of[(-rel).clamp(min=0)]
        if t:
            blocks = -(-lk // 32) * 4
            keep = _draws64((ident, step), np.arange(h * lq * blocks, dtype=np.uint64), 3)
            keep = keep.reshape(h, lq, blocks // 4, 4, 4, 2).transpose(0, 1, 2, 4, 3, 5).reshape(h, lq, blocks * 8)[:, :, :lk] >= t
            keep = torch.from_numpy(np.ascontiguousarray(keep)).to(DEV) * (65536.0 / (65536 - t))
        for c in range(h):
            sc = q[qs, c] @ k[ks, c // group].t() / math.sqrt(d) + table[:, c][bucket]
            if case["causal"]:
                sc = sc.masked_fill(rel > 0, -math.inf)
            p = torch.softmax(sc, dim=1)
            o = (p * keep[c] if t else p) @ v[ks, c // group]
            with torch.no_grad():
                out[qs, c] = o
                if case["train"]:
                    for total, one in zip(grads, torch.autograd.grad(o, (q, k, v, table), s["dout"][qs, c].double())):
                        total += one
    return {"out": out.detach(), **dict(zip(("dq", "dk", "dv", "dtable"), grads))} if case["train"] else out
