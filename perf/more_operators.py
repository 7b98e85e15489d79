"""The rest of the Boss's training step, as measured cases: linear layers with bias, activation and residual, layer normalisation, and AdamW
over many tensors.

``run`` computes each operator in its plain form (elementary torch operations in 32 bits, rounded once at the end) or, where ``own`` is
true, by the calls of ``paper_1905_03381_b200.binding``.  ``exact`` restates the definitions in 64 bits.

AdamW with states in 8 bits rounds them at random, without bias: sixteen bits of Philox4x32-10 for each moment of each element, keyed by
(seed, step, tensor, element), are part of its definition.  The states are e4m3 numbers in units of one power of two per 256 elements.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SEED = 20190503   # seed of the Philox draws
RULE = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.98, "eps": 1e-9}
DECAY = 0.01      # of matrices; vectors are not decayed


# ---------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one new token onto a vocabulary of 32,000 words: serving, the weights are all there is to read
        {"name": "linear_one_token_vocab", "op": "linear", "dtype": "bf16", "grad": False, "rows": 1, "inner": 512, "cols": 32000, "act": "none",
         "residual": False},
        # a feed-forward layer on one short sentence
        {"name": "linear_sentence_relu", "op": "linear", "dtype": "bf16", "grad": False, "rows": 17, "inner": 512, "cols": 2048, "act": "relu",
         "residual": False},
        # the second feed-forward layer on a translation batch of 25,000 tokens, with the block's residual connection
        {"name": "linear_ffn_forward", "op": "linear", "dtype": "bf16", "grad": False, "rows": 25000, "inner": 2048, "cols": 512, "act": "none",
         "residual": True},
        # gradients of the first feed-forward layer on the same batch
        {"name": "linear_ffn_grad", "op": "linear", "dtype": "bf16", "grad": True, "rows": 25000, "inner": 512, "cols": 2048, "act": "gelu",
         "residual": True},
        # gradients of the projection onto the vocabulary: the largest products of the step
        {"name": "linear_vocab_grad", "op": "linear", "dtype": "bf16", "grad": True, "rows": 25000, "inner": 512, "cols": 32000, "act": "none",
         "residual": False},
        # fp32 and odd widths, rows that start at every alignment
        {"name": "linear_f32_odd_grad", "op": "linear", "dtype": "f32", "grad": True, "rows": 4099, "inner": 515, "cols": 1001, "act": "silu",
         "residual": False},
        # one short sentence's activations
        {"name": "norm_one_sentence", "op": "norm", "dtype": "bf16", "grad": False, "rows": 17, "cols": 512, "residual": False},
        # backward pass of a normalisation inside a residual block of the translation batch
        {"name": "norm_translation_grad", "op": "norm", "dtype": "bf16", "grad": True, "rows": 25000, "cols": 512, "residual": True},
        # wide odd fp32 rows
        {"name": "norm_wide_odd_grad", "op": "norm", "dtype": "f32", "grad": True, "rows": 3001, "cols": 4099, "residual": False},
        # a small Boss of one layer: the call's latency
        {"name": "adamw_one_layer", "op": "adamw", "dtype": "f32", "bits": 32, "layers": 1, "width": 128, "inner": 512, "vocab": 1000, "copy": True},
        # the translation Boss's six layers, embedding and projection, fp32 moments
        {"name": "adamw_translation", "op": "adamw", "dtype": "bf16", "bits": 32, "layers": 6, "width": 512, "inner": 2048, "vocab": 32000, "copy": True},
        # the same with moments in 8 bits
        {"name": "adamw_translation_8bit", "op": "adamw", "dtype": "bf16", "bits": 8, "layers": 6, "width": 512, "inner": 2048, "vocab": 32000, "copy": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "norm", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "linear":
        rows = _log_int(rng, 1, 16) if rng.random() < 0.3 else _log_int(rng, 17, 32768)
        inner, cols = _log_int(rng, 64, 8192), _log_int(rng, 64, 32000)
        if rng.random() < 0.7:                     # widths of real layers; the rest are odd ones
            inner, cols = -(-inner // 64) * 64, -(-cols // 64) * 64
        room = (4.0e11 if dtype == "bf16" else 2.0e10) / (float(inner) * cols)
        rows = max(1, min(rows, int(room), 800_000_000 // cols))
        return {"op": op, "dtype": dtype, "grad": rng.random() < 0.5, "rows": rows, "inner": inner, "cols": cols,
                "act": rng.choice(["none", "relu", "gelu", "silu"]), "residual": rng.random() < 0.5}
    if op == "norm":
        cols = _log_int(rng, 64, 16384)
        if rng.random() < 0.7:
            cols = -(-cols // 64) * 64
        rows = _log_int(rng, 1, max(2, 12_000_000 // cols))
        return {"op": op, "dtype": dtype, "grad": rng.random() < 0.6, "rows": rows, "cols": cols, "residual": rng.random() < 0.5}
    width = 64 * rng.randint(1, 8)
    return {"op": op, "dtype": dtype, "bits": rng.choice([8, 32]), "layers": rng.randint(1, 6), "width": width, "inner": 4 * width,
            "vocab": _log_int(rng, 100, 32000), "copy": rng.random() < 0.7}


def _shapes(case):
    """Parameters of a translation Boss."""
    w, f = case["width"], case["inner"]
    layer = [(3 * w, w), (3 * w,), (w, w), (w,), (w,), (w,), (f, w), (f,), (w, f), (w,), (w,), (w,), (32, max(1, w // 64))]
    return [(case["vocab"], w)] + layer * case["layers"] + [(w,), (w,), (case["vocab"], w), (case["vocab"],)]


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        states = 16 if case["bits"] == 32 else 4 + 4 / 256
        return {"bytes": n * (8 + es + states + (2 if case["copy"] else 0)), "flops": 15.0 * n}
    m, n = case["rows"], case["cols"]
    if case["op"] == "norm":
        if case["grad"]:   # x, dout, the residual's gradient -> dx
            return {"bytes": m * n * es * (4 if case["residual"] else 3) + 12 * n, "flops": 14.0 * m * n}
        return {"bytes": 2 * m * n * es + 8 * n, "flops": 8.0 * m * n}
    k, act = case["inner"], case["act"] != "none"
    if case["grad"]:       # x, w, dout, pre, residual -> dx, dw, dbias
        elems = (3 if case["residual"] else 2) * m * k + 2 * n * k + (2 if act else 1) * m * n
        return {"bytes": elems * es + 4 * n, "flops": 4.0 * m * n * k}
    elems = m * k + n * k + (1 + act + case["residual"]) * m * n
    return {"bytes": elems * es + 4 * n, "flops": 2.0 * m * n * k}


# --------------------------------------------------------------------------------------------------------------- inputs

def _slots(case):
    """(first element, elements, whether it is decayed) of each tensor in the flat buffers; tensors start at multiples of 256."""
    got, at = [], 0
    for s in _shapes(case):
        n = math.prod(s)
        got.append((at, n, len(s) > 1))
        at += -(-n // 256) * 256
    return got, at


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(shape, std=1.0, t=dtype):
        return torch.randn(shape, generator=g, device=DEV).mul_(std).to(t)

    s = {"case": case}
    if case["op"] == "linear":
        m, k, n = case["rows"], case["inner"], case["cols"]
        s["x"], s["w"] = normal((m, k)), normal((n, k), k ** -0.5)
        if case["grad"]:
            s["dout"] = normal((m, n))
            s["pre"] = normal((m, n)) if case["act"] != "none" else None
            s["residual"] = normal((m, k)) if case["residual"] else None       # the gradient that reaches x past the layer
        else:
            s["bias"] = normal((n,), 0.1, torch.float32)
            s["residual"] = normal((m, n)) if case["residual"] else None
    elif case["op"] == "norm":
        m, n = case["rows"], case["cols"]
        s["x"] = (torch.randn((m, n), generator=g, device=DEV) * 1.5 + 0.3).to(dtype)
        s["gamma"] = normal((n,), 0.2, torch.float32) + 1.0
        if case["grad"]:
            s["dout"] = normal((m, n))
            s["residual"] = normal((m, n)) if case["residual"] else None
        else:
            s["beta"] = normal((n,), 0.2, torch.float32)
    else:
        slots, total = _slots(case)
        real = torch.zeros(total, dtype=torch.bool, device=DEV)
        for at, n, _ in slots:
            real[at:at + n] = True
        s["t"] = 1000
        s["param"] = normal((total,), 0.05, torch.float32) * real
        # gradients of unequal size along a tensor, moments that have seen such gradients
        size = torch.exp(torch.randn(total, generator=g, device=DEV) - 6.0) * real
        s["grad"] = (normal((total,), 1.0, torch.float32) * size).to(dtype)
        m = normal((total,), 0.3, torch.float32) * size
        root = (0.5 + torch.rand(total, generator=g, device=DEV)) * size
        if case["bits"] == 32:
            s["m"], s["v"] = m, root * root
        else:
            for name, x in (("m", m), ("root", root)):
                scale = _scale_of(x)
                s[name] = (x.view(-1, 256) / scale.float()[:, None]).reshape(-1).to(torch.float8_e4m3fn)
                s[name + "_scale"] = scale
        s["copy"] = s["param"].to(torch.bfloat16) if case["copy"] else None
    return s


def _scale_of(x):
    """Power of two per 256 elements that puts the largest of them into [128, 256)."""
    top = x.abs().view(-1, 256).amax(1)
    e = (top.view(torch.int32) >> 23) - 7
    return torch.where(top > 0, e.clamp(min=1), torch.zeros_like(e)).to(torch.uint8).view(torch.float8_e8m0fnu)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_1905_03381_b200 import binding as B
        s["aa"] = aa = B.AutoAssist(max_rows=1, max_d=16, device="cuda:0")
        if case["op"] == "linear":
            act = None if case["act"] == "none" else case["act"]
            s["activation"] = act
            if case["grad"]:
                s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
                s["dbias"] = torch.empty(case["cols"], device=DEV)
                s["scratch"] = aa.linear_grad_scratch(s["x"], s["w"], activation=act)
            else:
                s["out"] = torch.empty((case["rows"], case["cols"]), dtype=s["x"].dtype, device=DEV)
                s["pre"] = torch.empty_like(s["out"]) if act else None
        elif case["op"] == "norm":
            if case["grad"]:
                s["dx"] = torch.empty_like(s["x"])
                s["dgamma"], s["dbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["gamma"])
                s["scratch"] = aa.layer_norm_grad_scratch(s["x"])
            else:
                s["out"] = torch.empty_like(s["x"])
        else:
            s["rule"] = B.adamw_rule(t=s["t"], seed=SEED, **RULE)
            entries = []
            for at, n, matrix in _slots(case)[0]:
                cut = slice(at, at + n)
                block = slice(at // 256, at // 256 + -(-n // 256))
                copy = s["copy"][cut] if case["copy"] else None
                if case["bits"] == 32:
                    states = {"m": s["m"][cut], "v": s["v"][cut]}
                else:
                    states = {"m": s["m"][cut], "v": s["root"][cut], "m_scale": s["m_scale"][block], "v_scale": s["root_scale"][block]}
                entries.append(B.adamw_tensor(s["param"][cut], s["grad"][cut], copy=copy, weight_decay=DECAY if matrix else 0.0, **states))
            s["list"] = B.adamw_list(entries)
    elif case["op"] == "adamw":
        slots, total = _slots(case)
        s["decay"] = torch.zeros(total, device=DEV)
        s["tensor"] = torch.zeros(total // 4, dtype=torch.int64, device=DEV)
        s["first"] = torch.zeros(total // 4, dtype=torch.int64, device=DEV)
        for i, (at, n, matrix) in enumerate(slots):
            end = at + -(-n // 256) * 256
            s["decay"][at:at + n] = DECAY if matrix else 0.0
            s["tensor"][at // 4:end // 4] = i
            s["first"][at // 4:end // 4] = at // 4
    return s


# ----------------------------------------------------------------------------------------------------------- one pass

def run(state):
    s, case = state, state["case"]
    if own:
        return _run_own(s, case)
    if case["op"] == "adamw":
        return _plain_adamw(s, case)
    return _plain_linear(s, case) if case["op"] == "linear" else _plain_norm(s, case)


def _adamw_outputs(s, case):
    names = ("param", "copy") + (("m", "v") if case["bits"] == 32 else ("m", "root", "m_scale", "root_scale"))
    return {n: s[n] for n in names if s[n] is not None}


def _run_own(s, case):
    aa = s["aa"]
    if case["op"] == "linear":
        if case["grad"]:
            aa.aa_linear_grad(s["x"], s["w"], s["dout"], s["scratch"], dx=s["dx"], dw=s["dw"], dbias=s["dbias"], activation=s["activation"],
                              pre=s["pre"], residual=s["residual"])
            return {"dx": s["dx"], "dw": s["dw"], "dbias": s["dbias"]}
        aa.aa_linear(s["x"], s["w"], s["out"], bias=s["bias"], activation=s["activation"], residual=s["residual"], pre=s["pre"])
        return {"out": s["out"], "pre": s["pre"]}
    if case["op"] == "norm":
        if case["grad"]:
            aa.aa_layer_norm_grad(s["x"], s["dout"], s["dx"], s["scratch"], gamma=s["gamma"], residual=s["residual"], dgamma=s["dgamma"], dbeta=s["dbeta"])
            return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
        aa.aa_layer_norm(s["x"], s["out"], gamma=s["gamma"], beta=s["beta"])
        return s["out"]
    aa.aa_adamw(s["list"], s["rule"])
    return _adamw_outputs(s, case)


# --------------------------------------------------------------------------------------------------------- plain forms

EPS = 1e-5   # of the normalisation
ROOT_2 = math.sqrt(2.0)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros((), device=DEV))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z / ROOT_2))
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z / ROOT_2)) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig))


def _plain_linear(s, case):
    t, act = s["x"].dtype, case["act"]
    x, w = s["x"].float(), s["w"].float()
    if case["grad"]:
        g = s["dout"].float()
        if act != "none":
            g = g * _act_slope(s["pre"].float(), act)
        dx = g @ w
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        return {"dx": dx.to(t), "dw": (g.t() @ x).to(t), "dbias": g.sum(0)}
    z = x @ w.t() + s["bias"]
    out = _act(z, act)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return {"out": out.to(t), "pre": None if act == "none" else z.to(t)}


def _plain_norm(s, case):
    x, t = s["x"].float(), s["x"].dtype
    c = x - x.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    h = c * r
    if not case["grad"]:
        return (h * s["gamma"] + s["beta"]).to(t)
    d = s["dout"].float()
    g = d * s["gamma"]
    dx = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return {"dx": dx.to(t), "dgamma": (d * h).sum(0), "dbeta": d.sum(0)}


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


def _to_e4m3(x, u, squares):
    """x in units of its block's scale -> e4m3.  u: 16 random bits (int32).  Up where they reach the remainder, or where x^2 is above that part
    of the way from the lower neighbour's square to the upper one's, so that the stored number's square has the mean x^2."""
    a = x.abs()
    low = a < 2.0**-6                                        # below the normal numbers steps are equal: those of [2^-6, 2^-5)
    y = torch.where(low, a + 2.0**-6, a)
    bits = y.view(torch.int32)
    y = ((bits if squares else bits + (u << 4)) & ~0xFFFFF).view(torch.float32)
    if squares:
        z = ((bits & ~0xFFFFF) + 0x100000).view(torch.float32)
        z = torch.where(low, z - 2.0**-6, z)
    y = torch.where(low, y - 2.0**-6, y)
    if squares:
        return torch.where((a - y) * (a + y) > u.float() * 2.0**-16 * ((z - y) * (z + y)), z, y)
    return torch.where(x < 0, -y, y)


def _plain_adamw(s, case):
    t = s["t"] = s["t"] + 1
    b1, b2 = RULE["beta1"], RULE["beta2"]
    g = s["grad"].float()
    blocks = None
    if case["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        blocks = (-1, 256)
        m, root = ((s[n].float().view(blocks) * s[n + "_scale"].float()[:, None]).view(-1) for n in ("m", "root"))
        v = root * root
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + (g * g) * (1.0 - b2)
    step = m / (torch.sqrt(v * (1.0 / (1.0 - b2**t))) + RULE["eps"])
    p = s["param"] * (1.0 - RULE["lr"] * s["decay"].double()).float() - step * (RULE["lr"] / (1.0 - b1**t))
    s["param"].copy_(p)
    if s["copy"] is not None:
        s["copy"].copy_(p)
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return _adamw_outputs(s, case)
    root = torch.sqrt(v)
    block = torch.arange(g.numel() // 4, device=DEV) - s["first"]
    z = torch.zeros_like(block)
    words = torch.stack(_philox(block, s["tensor"], z + (t & _M32), z + (t >> 32), z + (SEED & _M32), z + (SEED >> 32)), 1).view(-1)
    for name, x, u in (("m", m, words & 0xFFFF), ("root", root, words >> 16)):
        scale = _scale_of(x)
        unit = scale.float()[:, None]
        unit = torch.where(unit < 2.0**-126, torch.ones((), device=DEV), unit)      # blocks of zeros
        code = _to_e4m3((x.view(blocks) / unit).view(-1), u.to(torch.int32), name == "root")
        if name == "root":
            code = torch.where((x > 0) & (code == 0), torch.full((), 2.0**-9, device=DEV), code)
        s[name].copy_(code.to(torch.float8_e4m3fn))
        s[name + "_scale"].copy_(scale)
    return _adamw_outputs(s, case)


# ------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s, case)
    x = s["x"].double().requires_grad_(case["grad"])
    if case["op"] == "norm":
        gamma = s["gamma"].double().requires_grad_(case["grad"])
        beta = torch.zeros_like(gamma, requires_grad=True) if case["grad"] else s["beta"].double()
        y = torch.nn.functional.layer_norm(x, (case["cols"],), gamma, beta, EPS)
        if not case["grad"]:
            return y
        dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), s["dout"].double())
        return {"dx": dx if s["residual"] is None else dx + s["residual"].double(), "dgamma": dgamma, "dbeta": dbeta}
    f = {"none": lambda z: z, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[case["act"]]
    if not case["grad"]:
        z = torch.addmm(s["bias"].double(), x, s["w"].double().t())
        out = f(z)
        return {"out": out if s["residual"] is None else out + s["residual"].double(), "pre": None if case["act"] == "none" else z}
    g = s["dout"].double()
    if case["act"] != "none":
        z = s["pre"].double().requires_grad_()
        (g,) = torch.autograd.grad(f(z), z, g)
    with torch.no_grad():
        dx = g @ s["w"].double()
        if s["residual"] is not None:
            dx += s["residual"].double()
        return {"dx": dx, "dw": torch.einsum("mn,mk->nk", g, x), "dbias": g.sum(0)}


def _draws64(blocks, tensor, t):
    """Words of the draws of one tensor's blocks of four elements (numpy)."""
    mask, mul = np.uint64(_M32), (np.uint64(0xD2511F53), np.uint64(0xCD9E8D57))
    one = np.ones(blocks, dtype=np.uint64)
    c = [np.arange(blocks, dtype=np.uint64), one * np.uint64(tensor), one * np.uint64(t & _M32), one * np.uint64(t >> 32)]
    k = [SEED % 2**32, SEED >> 32]
    for _ in range(10):
        a, b = mul[0] * c[0], mul[1] * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & mask, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & mask]
        k = [(k[0] + 0x9E3779B9) % 2**32, (k[1] + 0xBB67AE85) % 2**32]
    return np.stack(c, 1).reshape(-1)


def _exact_adamw(s, case):
    t, got = s["t"] + 1, {}
    lr, b1, b2, eps = (RULE[n] for n in ("lr", "beta1", "beta2", "eps"))
    slots, total = _slots(case)
    if case["bits"] == 8 and total > 120_000_000:
        return None
    unit = {n: s[n + "_scale"].double().repeat_interleave(256) for n in ("m", "root")} if case["bits"] == 8 else None
    g = s["grad"].double()
    m = s["m"].double() if unit is None else s["m"].double() * unit["m"]
    v = s["v"].double() if unit is None else (s["root"].double() * unit["root"]) ** 2
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    p = s["param"].double()
    for at, n, matrix in slots:
        if matrix:
            p[at:at + n] *= 1 - lr * DECAY
    p -= lr * (m / (1 - b1**t)) / (torch.sqrt(v / (1 - b2**t)) + eps)
    got["param"] = p
    if s["copy"] is not None:
        got["copy"] = p
    if unit is None:
        return {**got, "m": m, "v": v}
    words = np.concatenate([_draws64(-(-n // 256) * 64, i, t) for i, (_, n, _) in enumerate(slots)])
    words = torch.from_numpy(words.astype(np.int64)).to(DEV)
    for name, x, u in (("m", m, words % 65536), ("root", torch.sqrt(v), words // 65536)):
        rows = x.abs().view(-1, 256)
        top = rows.amax(1, keepdim=True)
        scale = torch.where(top > 0, 2.0 ** (torch.floor(torch.log2(top.clamp(min=1e-300))) - 7), torch.full_like(top, 2.0**-127))
        y = rows / scale
        step = 2.0 ** (torch.floor(torch.log2(y.clamp(min=2.0**-6))) - 3)            # e4m3 steps; equal ones below 2^-6
        u64 = u.view(-1, 256).double() / 65536
        if name == "m":
            code = torch.floor(y / step + u64) * step
        else:
            low = torch.floor(y / step) * step
            code = torch.where(y**2 - low**2 > u64 * ((low + step) ** 2 - low**2), low + step, low)
            code = torch.where((rows > 0) & (code == 0), torch.full_like(code, 2.0**-9), code)
        got[name] = (code * torch.sign(x.view(-1, 256))).view(-1)
        got[name + "_scale"] = scale[:, 0]
    return got
