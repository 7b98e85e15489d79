"""Linear layers, layer normalisation and AdamW against their fp64 reference.

Bars (derived from the formats, fixed before any run; a rounding is half a step: 2^-8 of a bf16 result, 2^-24 of an fp32 one):
  sums      : n terms in fp32, in any order, with roundings of at most a whole step: n 2^-23 of the sum of absolute terms, of which blocks of 16 count once on the
              matrix units.  fp32 operands are taken apart into terms whose products leave out less than 2^-22 of each product.  Together at most
              c(n) = 2^-21 + n 2^-24 (sequential sums round to nearest).
  activation: slopes are at most 1.13; erf, exp and quotients are good to a few 2^-24 of max(|z|, 1): 2^-20.
  bf16 G    : 2^-8 of each factor of the second products.
  norm      : a row's mean is off by at most 2^-18 mean|x| (sums of up to 40 terms a thread and a tree), so h by r 2^-18 mean|x| + 2^-18 |h|.
  AdamW     : about eight roundings a value: 2^-20 of the terms.  8-bit states: equal, code for code, to the formula in fp32 with every operation
              rounded by itself.
"""
import numpy as np
import pytest
import torch

import boss_step_reference as S
from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build, workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0**-24, BF16: 2.0**-8}


@pytest.fixture(scope="module")
def aa():
    build.build()
    ctx = B.AutoAssist(max_rows=1 << 10, max_d=64, device=DEV)
    yield ctx
    torch.cuda.synchronize()
    assert ctx.aa_device_status() == B.AA_OK
    ctx.close()


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def mat(rows, cols, seed, dtype, pad=0, shift=0, std=1.0):
    """rows x cols with `pad` columns behind each row and `shift` elements before the first."""
    flat = W.normal((rows * (cols + pad) + shift,), std, seed, dtype, DEV)
    return flat[shift:].view(rows, cols + pad)[:, :cols]


def like(shape, dtype, pad=0, fill=7.0):
    return torch.full((shape[0], shape[1] + pad), fill, dtype=dtype, device=DEV)[:, :shape[1]]


def close(got, want, bar):
    got = f64(got)
    assert got.shape == want.shape
    off = np.abs(got - want) - bar
    assert np.all(off <= 0), f"off by {np.abs(got - want).max():.3e}, {off.max():.3e} above the bar, at {np.unravel_index(off.argmax(), off.shape)}"


def c(n):
    return 2.0**-21 + n * 2.0**-24


# ------------------------------------------------------------------------------------------------------------------ linear

def check_linear(aa, dtype, m, k, n, act, bias, residual, pre, pads=(0, 0, 0), shift=0, **live):
    x, w = mat(m, k, 1, dtype, pads[0], shift), mat(n, k, 2, dtype, pads[1], shift, std=k ** -0.5)
    b = W.normal((n,), 0.5, 3, F32, DEV) if bias else None
    res = mat(m, n, 4, dtype, pads[2], shift) if residual else None
    out, p = like((m, n), dtype, pads[2]), like((m, n), dtype, pads[2]) if pre else None
    aa.aa_linear(x, w, out, bias=b, activation=act, residual=res, pre=p, **live)
    want, z, size = S.linear(f64(x), f64(w), f64(b), act, f64(res))
    bar = 1.13 * c(k) * size + 2.0**-20 * np.maximum(np.abs(z), 1.0) * (act is not None) + HALF[dtype] * np.abs(want) + 2.0**-22 * np.abs(z)
    return out, p, want, z, bar, c(k) * size + HALF[dtype] * np.abs(z)


SHAPES = [(1, 1, 1), (1, 512, 2048), (2, 64, 1000), (3, 7, 5), (8, 1000, 129), (16, 512, 512), (17, 512, 2048), (33, 65, 31), (64, 64, 64), (100, 72, 264), (127, 96, 257),
          (129, 520, 128), (257, 40, 300), (300, 2048, 64), (1000, 136, 520), (40, 5000, 24)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear_of_many_sizes(aa, dtype, m, k, n):
    out, p, want, z, bar, pre_bar = check_linear(aa, dtype, m, k, n, "gelu", True, True, True)
    close(out, want, bar)
    close(p, z, pre_bar)
    out, _, want, _, bar, _ = check_linear(aa, dtype, m, k, n, None, False, False, False)
    close(out, want, bar)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", [None, "relu", "gelu", "silu"])
@pytest.mark.parametrize("m", [5, 150])
def test_linear_activations_and_optional_operands(aa, dtype, act, m):
    for bias, residual, pre in ((True, False, True), (False, True, False), (True, True, True)):
        out, p, want, z, bar, pre_bar = check_linear(aa, dtype, m, 96, 200, act, bias, residual, pre)
        close(out, want, bar)
        if pre:
            close(p, z, pre_bar)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pads,shift", [((8, 16, 24), 0), ((3, 5, 1), 0), ((1, 0, 0), 1), ((0, 0, 3), 3), ((4, 4, 4), 4)])
@pytest.mark.parametrize("m", [6, 140])
def test_linear_strides_and_alignment(aa, dtype, pads, shift, m):
    out, p, want, z, bar, pre_bar = check_linear(aa, dtype, m, 120, 136, "silu", True, True, True, pads, shift)
    close(out, want, bar)
    close(p, z, pre_bar)
    behind = out.as_strided((m - 1, pads[2]), (out.stride(0), 1), out.storage_offset() + 136)
    assert torch.all(behind == 7.0)


def live_forms():
    """(rows evaluated of 300, arguments)."""
    off = i32([0, 10, 10, 137, 290])
    return [(300, {}), (131, {"count_dev": i32([131])}), (0, {"count_dev": i32([-3])}), (300, {"count_dev": i32([400])}), (290, {"offsets": off}),
            (137, {"offsets": off, "count_dev": i32([3])}), (10, {"offsets": off, "count_dev": i32([2])}), (0, {"offsets": off, "count_dev": i32([0])}), (290, {"offsets": off, "count_dev": i32([9])})]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("form", range(9))
def test_linear_of_counted_rows(aa, dtype, form):
    rows, live = live_forms()[form]
    x, w, res, dout, pre = (mat(a, b, s, dtype) for a, b, s in ((300, 104, 1), (72, 104, 2), (300, 72, 3), (300, 72, 4), (300, 72, 5)))
    for t in (x, res, dout, pre):
        t[rows:] = float("nan")                 # what is not evaluated may hold anything
    out = like((300, 72), dtype)
    aa.aa_linear(x, w, out, residual=res, **live)
    want, z, size = S.linear(f64(x)[:rows], f64(w), None, None, f64(res)[:rows])
    close(out[:rows], want, c(104) * size + HALF[dtype] * np.abs(want) + 2.0**-22 * np.abs(z))
    assert torch.all(out[rows:] == 7.0)
    for act in (None, "relu"):
        dx, dw, db = like((300, 104), dtype), like((72, 104), dtype), torch.full((72,), 7.0, device=DEV)
        aa.aa_linear_grad(x, w, dout, aa.linear_grad_scratch(x, w, act), dx=dx, dw=dw, dbias=db, activation=act, pre=None if act is None else pre, **live)
        got, size, _ = S.linear_grad(f64(x)[:rows], f64(w), f64(dout)[:rows], act, f64(pre)[:rows], None)
        close(dx[:rows], got["dx"], c(72) * size["dx"] + HALF[dtype] * np.abs(got["dx"]))
        assert torch.all(dx[rows:] == 7.0)
        close(dw, got["dw"], c(rows) * size["dw"] + HALF[dtype] * np.abs(got["dw"]))
        close(db, got["dbias"], c(rows) * size["dbias"])


def check_grad(aa, dtype, m, k, n, act, residual, pads=(0, 0, 0), shift=0, which=("dx", "dw", "dbias")):
    x, w, dout = mat(m, k, 1, dtype, pads[0], shift), mat(n, k, 2, dtype, pads[1], shift, std=k ** -0.5), mat(m, n, 3, dtype, pads[2], shift)
    pre = mat(m, n, 4, dtype, pads[2], shift) if act else None
    res = mat(m, k, 5, dtype, pads[0], shift) if residual else None
    outs = {"dx": like((m, k), dtype, pads[0]), "dw": like((n, k), dtype, pads[1]), "dbias": torch.full((n,), 7.0, device=DEV)}
    outs = {name: outs[name] for name in which}
    scratch = aa.linear_grad_scratch(x, w, act)
    aa.aa_linear_grad(x, w, dout, scratch, activation=act, pre=pre, residual=res, **outs)
    got, size, g = S.linear_grad(f64(x), f64(w), f64(dout), act, f64(pre), f64(res))
    slope = 2.0**-20 * np.abs(f64(dout)) * (act not in (None, "relu"))       # absolute error of G
    rounded = 2.0**-8 if dtype == BF16 and act not in (None, "relu") else 0.0
    bars = {"dx": (c(n) + rounded) * size["dx"] + slope @ np.abs(f64(w)), "dw": (c(m) + rounded) * size["dw"] + slope.T @ np.abs(f64(x)),
            "dbias": c(m) * size["dbias"] + slope.sum(0)}
    for name, t in outs.items():
        bar = bars[name] + (HALF[dtype] * np.abs(got[name]) if name != "dbias" else 0.0) + 2.0**-22 * np.abs(got[name])
        close(t, got[name], bar)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear_gradients_of_many_sizes(aa, dtype, m, k, n):
    check_grad(aa, dtype, m, k, n, "gelu", True)
    check_grad(aa, dtype, m, k, n, None, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", [None, "relu", "gelu", "silu"])
def test_linear_gradients_alone_and_together(aa, dtype, act):
    for which in (("dx",), ("dw",), ("dbias",), ("dx", "dbias"), ("dw", "dbias"), ("dx", "dw")):
        check_grad(aa, dtype, 150, 96, 200, act, "dx" in which, which=which)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pads,shift", [((8, 16, 24), 0), ((3, 5, 1), 0), ((1, 0, 0), 1), ((0, 0, 3), 3)])
def test_linear_gradients_strides_and_alignment(aa, dtype, pads, shift):
    check_grad(aa, dtype, 140, 120, 136, "silu", True, pads, shift)
    check_grad(aa, dtype, 140, 120, 136, None, True, pads, shift)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_linear_in_place_residuals(aa, dtype):
    x, w, res = mat(130, 64, 1, dtype), mat(72, 64, 2, dtype), mat(130, 72, 3, dtype)
    one, two = torch.empty_like(res), res.clone()
    aa.aa_linear(x, w, one, residual=res)
    aa.aa_linear(x, w, two, residual=two)
    assert torch.equal(one, two)
    dres = mat(130, 64, 4, dtype)
    one, two, scratch = torch.empty_like(dres), dres.clone(), aa.linear_grad_scratch(x, w)
    aa.aa_linear_grad(x, w, res, scratch, dx=one, residual=dres)
    aa.aa_linear_grad(x, w, res, scratch, dx=two, residual=two)
    assert torch.equal(one, two)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m", [4, 200])
def test_linear_gradient_against_differences(aa, dtype, m):
    """The directional derivative of sum(out * t) along one direction of x, w and bias, by central differences in fp64 of the reference and by the call."""
    x, w, t = mat(m, 40, 1, dtype), mat(24, 40, 2, dtype, std=0.2), mat(m, 24, 3, dtype)
    b = W.normal((24,), 0.5, 4, F32, DEV)
    pre, out = like((m, 24), dtype), like((m, 24), dtype)
    aa.aa_linear(x, w, out, bias=b, activation="gelu", pre=pre)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    aa.aa_linear_grad(x, w, t, aa.linear_grad_scratch(x, w, "gelu"), dx=dx, dw=dw, dbias=db, activation="gelu", pre=pre)
    rng = np.random.default_rng(1)
    ux, uw, ub = (rng.standard_normal(tuple(v.shape)) for v in (x, w, b))
    f = lambda e: (S.linear(f64(x) + e * ux, f64(w) + e * uw, f64(b) + e * ub, "gelu", None)[0] * f64(t)).sum()  # noqa: E731
    want = (f(1e-5) - f(-1e-5)) / 2e-5
    got = (f64(dx) * ux).sum() + (f64(dw) * uw).sum() + (f64(db) * ub).sum()
    size = np.abs(f64(dx) * ux).sum() + np.abs(f64(dw) * uw).sum() + np.abs(f64(db) * ub).sum()
    # roundings of the three gradients, of G and of pre (which moves slopes of at most 0.8 a unit)
    assert abs(got - want) <= (4 * HALF[dtype] + 2.0**-14) * size


def test_linear_infinities_and_nans_stay_in_their_rows(aa):
    for dtype in (F32, BF16):
        for m in (7, 140):
            x, w = mat(m, 64, 1, dtype), mat(40, 64, 2, dtype)
            x[2, 5], x[4, 9] = float("inf"), float("nan")
            out = like((m, 40), dtype)
            aa.aa_linear(x, w, out, activation="relu")
            clean = torch.ones(m, dtype=torch.bool, device=DEV)
            clean[2] = clean[4] = False
            want, z, size = S.linear(f64(x[clean]), f64(w), None, "relu", None)
            close(out[clean], want, c(64) * size + HALF[dtype] * np.abs(want) + 2.0**-20)
            assert torch.all(torch.isnan(out[4]))
            assert not torch.any(torch.isfinite(out[2]) & (out[2] != 0))


def refused(call, status=B.AA_ERR_INVALID_ARG):
    with pytest.raises(B.AutoAssistError) as e:
        call()
    assert e.value.status == status


def test_linear_refusals(aa):
    x, w, out = mat(10, 16, 1, F32), mat(8, 16, 2, F32), like((10, 8), F32)
    refused(lambda: aa.aa_linear(x, w, like((10, 7), F32)))
    refused(lambda: aa.aa_linear(x, w, like((9, 8), F32)))
    refused(lambda: aa.aa_linear(x, w, like((10, 8), BF16)))
    refused(lambda: aa.aa_linear(x, mat(8, 15, 2, F32), out))
    refused(lambda: aa.aa_linear(x, w.bfloat16(), out))
    refused(lambda: aa.aa_linear(x, w, out, residual=like((10, 9), F32)))
    refused(lambda: aa.aa_linear(x, w, out, pre=out))
    refused(lambda: aa.aa_linear(x, w, x[:, :8]))
    flat = torch.zeros(200, device=DEV)
    refused(lambda: aa.aa_linear(x, w, flat[:80].view(10, 8), residual=flat[8:88].view(10, 8)))
    for bad in (lambda: aa.aa_linear(x, w, out, bias=torch.zeros(7, device=DEV)), lambda: aa.aa_linear(x, w, out, activation="tanh"),
                lambda: aa.aa_linear(x, w, out, bias=torch.zeros(8, dtype=BF16, device=DEV)), lambda: aa.aa_linear(x, w, out, offsets=i32([0, 3]), n_seg=2)):
        with pytest.raises(TypeError):
            bad()
    s = aa.linear_grad_scratch(x, w)
    dout, dx, dw = like((10, 8), F32), like((10, 16), F32), like((8, 16), F32)
    refused(lambda: aa.aa_linear_grad(x, w, dout, s, dx=dx, pre=dout))
    refused(lambda: aa.aa_linear_grad(x, w, dout, s, dx=dx, activation="relu"))
    refused(lambda: aa.aa_linear_grad(x, w, dout, s, dw=dw, residual=dx))
    refused(lambda: aa.aa_linear_grad(x, w, dout, s, dx=x))
    refused(lambda: aa.aa_linear_grad(x, w, dout, s, dw=w))
    refused(lambda: aa.aa_linear_grad(x, w, dout, s, dx=like((10, 15), F32)))
    refused(lambda: aa.aa_linear_grad(x, w, dout, s[:300], dx=dx), B.AA_ERR_WORKSPACE)
    aa.aa_linear(x, w, out, offsets=i32([0, 11]))
    torch.cuda.synchronize()
    assert aa.aa_device_status() == B.AA_ERR_BAD_INDEX and torch.all(out == 7.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_no_rows_are_zero(aa, dtype):
    x, w = torch.zeros((0, 24), dtype=dtype, device=DEV), mat(16, 24, 1, dtype)
    dw, db = like((16, 24), dtype), torch.full((16,), 7.0, device=DEV)
    aa.aa_linear_grad(x, w, torch.zeros((0, 16), dtype=dtype, device=DEV), aa.linear_grad_scratch(x, w), dw=dw, dbias=db)
    assert torch.all(dw == 0) and torch.all(db == 0)
    aa.aa_linear(x, w, torch.zeros((0, 16), dtype=dtype, device=DEV))
    dg, db = torch.full((24,), 7.0, device=DEV), torch.full((24,), 7.0, device=DEV)
    aa.aa_layer_norm_grad(x, x, x.clone(), aa.layer_norm_grad_scratch(x), dgamma=dg, dbeta=db)
    assert torch.all(dg == 0) and torch.all(db == 0)


# ---------------------------------------------------------------------------------------------------------------------- norm

def norm_bars(x, h, r, dtype):
    e = 2.0**-18 * (1.0 + np.abs(h)) + r * 2.0**-18 * np.abs(x).mean(1, keepdims=True)       # of h
    return e


def check_norm(aa, dtype, m, n, pad=0, shift=0, eps=1e-5, affine=True, residual=True, offset=0.3, inplace=False):
    x = mat(m, n, 1, dtype, pad, shift)
    x.mul_(1.5).add_(offset)
    gamma, beta = (W.normal((n,), 0.3, s, F32, DEV) + s for s in (1, 0)) if affine else (None, None)
    out = x.clone() if inplace else like((m, n), dtype, pad)
    aa.aa_layer_norm(out if inplace else x, out, gamma=gamma, beta=beta, eps=eps)
    want, h, r = S.layer_norm(f64(x), f64(gamma), f64(beta), eps)
    e = norm_bars(f64(x), h, r, dtype)
    scale = 1.0 if gamma is None else np.abs(f64(gamma))
    close(out, want, scale * e + HALF[dtype] * np.abs(want) + 2.0**-22 * np.abs(want))
    d, res = mat(m, n, 2, dtype, pad, shift), mat(m, n, 3, dtype, pad, shift) if residual else None
    dx = d.clone() if inplace else like((m, n), dtype, pad)
    dg, db = torch.full((n,), 7.0, device=DEV), torch.full((n,), 7.0, device=DEV)
    aa.aa_layer_norm_grad(x, dx if inplace else d, dx, aa.layer_norm_grad_scratch(x), gamma=gamma, eps=eps, residual=res, dgamma=dg, dbeta=db)
    got, h, r, g = S.layer_norm_grad(f64(x), f64(gamma), eps, f64(d), f64(res))
    mg, mgh = np.abs(g).mean(1, keepdims=True), np.abs(g * h).mean(1, keepdims=True)
    bar = r * (2.0**-18 * (np.abs(g) + mg) + e * (mgh + mg) + np.abs(h) * ((np.abs(g) * e).mean(1, keepdims=True) + 2.0**-18 * mgh)) + 2.0**-17 * np.abs(got["dx"])
    close(dx, got["dx"], bar + HALF[dtype] * np.abs(got["dx"]))
    close(dg, got["dgamma"], (np.abs(f64(d)) * e).sum(0) + c(m) * np.abs(f64(d) * h).sum(0))
    close(db, got["dbeta"], c(m) * np.abs(f64(d)).sum(0))


NORM = [(1, 1), (3, 2), (7, 63), (5, 64), (40, 100), (33, 128), (17, 200), (300, 256), (17, 512), (2000, 512), (9, 513), (50, 1000), (21, 2048), (70, 4096), (6, 4099), (11, 8192),
        (3, 8193), (5, 20001)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n", NORM)
def test_norm_of_many_sizes(aa, dtype, m, n):
    check_norm(aa, dtype, m, n)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (0, 1), (3, 5)])
@pytest.mark.parametrize("n", [96, 520, 3000])
def test_norm_strides_and_alignment(aa, dtype, pad, shift, n):
    check_norm(aa, dtype, 19, n, pad, shift)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [64, 1000, 9000])
def test_norm_without_weights_far_means_and_in_place(aa, dtype, n):
    check_norm(aa, dtype, 12, n, affine=False, residual=False)
    check_norm(aa, dtype, 12, n, offset=100.0)
    check_norm(aa, dtype, 12, n, inplace=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_of_constant_rows(aa, dtype):
    """Variance 0: h is 0 and the gradient's scale is 1 / sqrt(eps)."""
    x, d = torch.full((5, 96), 3.0, dtype=dtype, device=DEV), mat(5, 96, 2, dtype)
    out, dx = torch.empty_like(x), torch.empty_like(x)
    beta = W.normal((96,), 1.0, 3, F32, DEV)
    aa.aa_layer_norm(x, out, beta=beta, eps=1e-2)
    close(out, np.broadcast_to(f64(beta), (5, 96)), HALF[dtype] * np.abs(f64(beta)) + 0 * f64(x))
    aa.aa_layer_norm_grad(x, d, dx, aa.layer_norm_grad_scratch(x), eps=1e-2)
    want = 10.0 * (f64(d) - f64(d).mean(1, keepdims=True))
    close(dx, want, HALF[dtype] * np.abs(want) + 2.0**-17)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [128, 1024, 8200])
@pytest.mark.parametrize("form", range(9))
def test_norm_of_counted_rows(aa, dtype, n, form):
    rows, live = live_forms()[form]
    x, d = mat(300, n, 1, dtype), mat(300, n, 2, dtype)
    x[rows:] = float("nan")
    d[rows:] = float("nan")
    out, dx = like((300, n), dtype), like((300, n), dtype)
    dg, db = torch.full((n,), 7.0, device=DEV), torch.full((n,), 7.0, device=DEV)
    aa.aa_layer_norm(x, out, **live)
    aa.aa_layer_norm_grad(x, d, dx, aa.layer_norm_grad_scratch(x), dgamma=dg, dbeta=db, **live)
    assert torch.all(out[rows:] == 7.0) and torch.all(dx[rows:] == 7.0)
    got, h, r, _ = S.layer_norm_grad(f64(x)[:rows], None, 1e-5, f64(d)[:rows], None)
    e = norm_bars(f64(x)[:rows], h, r, dtype)
    close(out[:rows], h, e + HALF[dtype] * np.abs(h))
    close(dg, got["dgamma"], (np.abs(f64(d)[:rows]) * e).sum(0) + c(rows) * np.abs(f64(d)[:rows] * h).sum(0))
    close(db, got["dbeta"], c(rows) * np.abs(f64(d)[:rows]).sum(0))


def test_norm_refusals(aa):
    x, v = mat(10, 16, 1, F32), torch.zeros(16, device=DEV)
    refused(lambda: aa.aa_layer_norm(x, like((10, 15), F32)))
    refused(lambda: aa.aa_layer_norm(x, like((10, 16), BF16)))
    refused(lambda: aa.aa_layer_norm(x, torch.empty_like(x), eps=-1.0))
    refused(lambda: aa.aa_layer_norm(x, torch.empty_like(x), eps=float("nan")))
    flat = torch.zeros(200, device=DEV)
    refused(lambda: aa.aa_layer_norm(flat[:160].view(10, 16), flat[16:176].view(10, 16)))
    s = aa.layer_norm_grad_scratch(x)
    refused(lambda: aa.aa_layer_norm_grad(x, x, torch.empty_like(x), s, dgamma=v, dbeta=v))
    refused(lambda: aa.aa_layer_norm_grad(x, x, torch.empty_like(x), s, gamma=v, dgamma=v))
    refused(lambda: aa.aa_layer_norm_grad(x, like((9, 16), F32), torch.empty_like(x), s))
    refused(lambda: aa.aa_layer_norm_grad(x, x, torch.empty_like(x), s[:300]), B.AA_ERR_WORKSPACE)
    with pytest.raises(TypeError):
        aa.aa_layer_norm(x, torch.empty_like(x), gamma=torch.zeros(15, device=DEV))


# --------------------------------------------------------------------------------------------------------------------- AdamW

RULE = {"lr": 2e-3, "beta1": 0.9, "beta2": 0.98, "eps": 1e-9}
E4M3 = None


def values(codes):
    global E4M3
    if E4M3 is None:
        E4M3 = S.e4m3_values()
    return E4M3[codes.view(torch.uint8).cpu().numpy()]


def entry(n, seed, grad_dtype, bits, copy, decay, shift=0):
    cut = lambda t: t[shift:]  # noqa: E731
    p, g = cut(W.normal((n + shift,), 0.1, seed, F32, DEV)), cut(W.normal((n + shift,), 1e-2, seed + 1, F32, DEV) * torch.exp(W.normal((n + shift,), 2.0, seed + 2, F32, DEV)))
    g = cut(torch.cat([torch.zeros(shift, device=DEV), g]).to(grad_dtype))
    k = {"copy": cut(torch.zeros(n + shift, dtype=BF16, device=DEV)) if copy else None, "weight_decay": decay}
    if bits == 32:
        k["m"], k["v"] = cut(W.normal((n + shift,), 1e-3, seed + 3, F32, DEV)), cut(W.normal((n + shift,), 1e-3, seed + 4, F32, DEV).square())
    else:
        m8 = B.adamw_moments8(torch.empty(n + shift, device=DEV))
        k.update({name: cut(m8[name]) for name in ("m", "v")})
        k.update({name: torch.zeros((n + 255) // 256, dtype=torch.uint8, device=DEV) for name in ("m_scale", "v_scale")})
    return B.adamw_tensor(p, g, **k)


SIZES = [1, 3, 255, 256, 257, 4095, 4096, 5000, 100_003]


@pytest.mark.parametrize("grad_dtype", [F32, BF16])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw_with_fp32_moments(aa, grad_dtype, shift):
    es = [entry(n, 10 * i, grad_dtype, 32, i % 2 == 0, 0.05 * (i % 3), shift) for i, n in enumerate(SIZES)]
    before = [[f64(t) for t in e._keep[:4]] for e in es]
    rule, table = B.adamw_rule(t=4, **RULE), B.adamw_list(es)
    for _ in range(2):
        aa.aa_adamw(table, rule)
    assert rule.t == 6
    for e, (p, g, m, v), i in zip(es, before, range(99)):
        size = np.abs(p)
        for t in (5, 6):
            p, m, v = S.adamw(p, g, m, v, {**RULE, "t": t}, 0.05 * (i % 3))
            size = size + RULE["lr"] * np.abs(m / 0.4) / (np.sqrt(v) + 1e-12)
        m_size = np.abs(before[i][2]) + np.abs(g)
        close(e._keep[2], m, 2.0**-21 * m_size)
        close(e._keep[3], v, 2.0**-20 * v)
        # m / sqrt(v) carries the terms m came from
        bar = 2.0**-20 * (size + RULE["lr"] * m_size / 0.4 / (np.sqrt(v) + 1e-12))
        close(e._keep[0], p, bar)
        if e._keep[6] is not None:
            assert torch.equal(e._keep[6], e._keep[0].to(BF16))


@pytest.mark.parametrize("grad_dtype", [F32, BF16])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw_with_8_bit_moments_code_for_code(aa, grad_dtype, shift):
    seed, es = 2**40 + 77, [entry(n, 10 * i, grad_dtype, 8, i % 2 == 0, 0.05 * (i % 3), shift) for i, n in enumerate(SIZES)]
    rule, table = B.adamw_rule(t=2**33, seed=seed, **RULE), B.adamw_list(es)
    for rep in range(3):
        before = [(e._keep[0].cpu().numpy(), e._keep[1].float().cpu().numpy(), *[(values(t) * np.repeat(np.where(s > 0, 2.0 ** (s - 127.0), 0), 256)[:len(t)]).astype(np.float32) for t, s in
                   ((e._keep[2], e._keep[4].cpu().numpy().astype(float)), (e._keep[3], e._keep[5].cpu().numpy().astype(float)))]) for e in es]
        aa.aa_adamw(table, rule)
        for i, (e, (p, g, m, root)) in enumerate(zip(es, before)):
            t = 2**33 + rep + 1
            p, m, v = S.adamw(p, g, m, root * root, {**RULE, "t": t}, 0.05 * (i % 3))
            assert p.dtype == m.dtype == v.dtype == np.float32
            for x, u, codes, scales, positive in zip((m, np.sqrt(v)), S.draws(len(m), seed, i, t), e._keep[2:4], e._keep[4:6], (False, True)):
                want, byte, units, step = S.to_codes(x, u, positive)
                assert np.array_equal(scales.cpu().numpy(), byte)
                got = values(codes)
                assert np.all(np.abs(np.abs(got) - units) <= np.where(np.abs(got) == 2.0**-9, 2.0**-9, step))      # a neighbour
                assert np.array_equal(got, want)
            assert np.max(np.abs(e._keep[0].cpu().numpy() - p) - 2.0**-22 * (np.abs(p) + RULE["lr"] * np.abs(m) / (np.sqrt(v) + 1e-9))) <= 0


def test_8_bit_moments_follow_a_constant_gradient_without_bias(aa):
    """With a constant gradient both moments approach it although most steps move them by less than half a code.  m and the square of root are unbiased,
    and an element's standard deviation stays below its mean (a step of drift d jumps by a code c <= 2^-3 with probability d / c, which sums to less than
    c / 2 in variance), so the mean over 65,536 of them is off by 5 / 256 at most (5 standard deviations)."""
    n = 65536
    p, g = torch.zeros(n, device=DEV), torch.full((n,), 0.37, device=DEV)
    e = B.adamw_tensor(p, g, **B.adamw_moments8(p))
    rule, table = B.adamw_rule(lr=0.0, beta1=0.9, beta2=0.99, seed=5), B.adamw_list([e])
    for _ in range(600):
        aa.aa_adamw(table, rule)
    m, root = (values(codes) * np.repeat(2.0 ** (scales.cpu().numpy().astype(float) - 127), 256) for codes, scales in ((e._keep[2], e._keep[4]), (e._keep[3], e._keep[5])))
    assert abs(m.mean() / (0.37 * (1 - 0.9**600)) - 1) <= 5 / 256
    assert abs((root**2).mean() / (0.37**2 * (1 - 0.99**600)) - 1) <= 5 / 256


def test_adamw_moments_of_zeros_and_tiny_numbers(aa):
    n = 700
    for bits in (8, 32):
        p, g = torch.ones(n, device=DEV), torch.zeros(n, device=DEV)
        g[300:310] = torch.tensor([1e-30, 1e-25, 1e-12, 1e-3, 1.0, 1e4, -1e-30, -1e-12, -1.0, 1e-38], device=DEV)
        k = B.adamw_moments8(p) if bits == 8 else {"m": torch.zeros(n, device=DEV), "v": torch.zeros(n, device=DEV)}
        e = B.adamw_tensor(p, g, **k)
        rule, table = B.adamw_rule(lr=1e-2, eps=1e-12), B.adamw_list([e])
        for _ in range(4):
            aa.aa_adamw(table, rule)
        got = f64(p)
        assert np.all(np.isfinite(got))
        assert np.all(got[np.r_[0:300, 310:700]] == 1.0)
        # no element is moved faster than a first step moves it, by more than a rounded code's half
        assert np.all(np.abs(got - 1.0) <= 4 * 1e-2 * 1.5)
        if bits == 8:
            root = values(e._keep[3])
            assert np.all(root[[303, 304, 305, 308]] > 0) and np.all(root[:256] == 0)


def test_adamw_grad_scale_and_skipped_steps(aa):
    for bits in (32, 8):
        one, two = (entry(3000, 5, F32, bits, True, 0.1) for _ in range(2))
        scaled = (two._keep[1] * 0.25).contiguous()
        k = dict(zip(("m", "v", "m_scale", "v_scale", "copy"), two._keep[2:]))
        two = B.adamw_tensor(two._keep[0], scaled, weight_decay=0.1, **k)
        aa.aa_adamw(B.adamw_list([one]), B.adamw_rule(**RULE), grad_scale=torch.tensor([0.25], device=DEV))
        aa.aa_adamw(B.adamw_list([two]), B.adamw_rule(**RULE))
        for a, b, i in zip(one._keep, two._keep, range(7)):
            assert a is None or i == 1 or torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        kept = [None if t is None else t.clone() for t in one._keep]
        for bad in (float("nan"), float("inf"), -float("inf")):
            aa.aa_adamw(B.adamw_list([one]), B.adamw_rule(**RULE), grad_scale=torch.tensor([bad], device=DEV))
        for a, b in zip(one._keep, kept):
            assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_adamw_long_lists_of_both_kinds(aa):
    """More tensors than a launch takes, both kinds of moments in turn: every tensor is updated once, by its own place in the list."""
    es = [entry(1 + 37 * (i % 11), i, BF16, 8 if i % 3 else 32, False, 0.01) for i in range(900)]
    before = [[t.clone() for t in e._keep[:2]] + [values(e._keep[2]) if e.state_bits == 8 else f64(e._keep[2])] for e in es]
    aa.aa_adamw(B.adamw_list(es), B.adamw_rule(seed=3, **RULE))
    for i in (0, 1, 2, 31, 254, 255, 256, 257, 300, 599, 600, 767, 768, 899):
        e, (p, g, m) = es[i], before[i]
        gg = f64(g)
        if e.state_bits == 8:
            want, byte, _, _ = S.to_codes(np.float32(1.0 - 0.9) * gg.astype(np.float32), S.draws(len(gg), 3, i, 1)[0], False)
            assert np.array_equal(values(e._keep[2]), want) and np.array_equal(e._keep[4].cpu().numpy(), byte)
        else:
            close(e._keep[2], 0.9 * m + 0.1 * gg, 2.0**-21 * (np.abs(m) + np.abs(gg)))
        assert not torch.equal(e._keep[0], p)


def test_adamw_refusals(aa):
    p, g, m, v = (torch.zeros(64, device=DEV) for _ in range(4))
    good = B.adamw_list([B.adamw_tensor(p, g, m, v)])
    for k in ({"lr": -1.0}, {"lr": float("nan")}, {"lr": 0.1, "beta1": 1.0}, {"lr": 0.1, "beta2": -0.1}, {"lr": 0.1, "eps": -1.0}, {"lr": 0.1, "t": -1}):
        rule = B.adamw_rule(**k)
        refused(lambda: aa.aa_adamw(good, rule))
        assert rule.t == k.get("t", 0)
    refused(lambda: aa.aa_adamw(B.adamw_list([B.adamw_tensor(p, g, m, v, weight_decay=float("inf"))]), B.adamw_rule(0.1)))
    for bad in (lambda: B.adamw_tensor(p, g[:63], m, v), lambda: B.adamw_tensor(p.bfloat16(), g, m, v), lambda: B.adamw_tensor(p, g, m, v, m_scale=torch.zeros(1, dtype=torch.uint8, device=DEV)),
                lambda: B.adamw_tensor(p, g, m.bfloat16(), v), lambda: B.adamw_list([B.adamw_tensor(p, g, m, v), B.adamw_tensor(v, g, p, m)]),
                lambda: B.adamw_list([B.adamw_tensor(p, p, m, v)])):
        with pytest.raises(TypeError):
            bad()
    raw = B.adamw_tensor(p, g, m, v)
    raw.v = m.data_ptr()
    table = (B.aa_adamw_tensor * 1)(raw)
    refused(lambda: aa.aa_adamw(table, B.adamw_rule(0.1)))
    raw.v, raw.state_bits = v.data_ptr(), 16
    table = (B.aa_adamw_tensor * 1)(raw)
    refused(lambda: aa.aa_adamw(table, B.adamw_rule(0.1)))
    # gradients may be shared, empty tensors and lists do nothing
    other = [torch.zeros(64, device=DEV) for _ in range(3)]
    none = torch.zeros(0, device=DEV)
    rule = B.adamw_rule(0.1)
    aa.aa_adamw(B.adamw_list([B.adamw_tensor(p, g, m, v), B.adamw_tensor(other[0], g, other[1], other[2]), B.adamw_tensor(none, none, none, none)]), rule)
    aa.aa_adamw(B.adamw_list([]), rule)
    assert rule.t == 2


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k,n", [(20, 4096, 64), (130, 1024, 200), (33, 8192, 130), (70, 2056, 24), (300, 513, 65), (17, 1001, 333), (200, 600, 1000)])
def test_linear_of_few_tiles_and_long_sums(aa, dtype, m, k, n):
    """Products that a few tiles cover and whose sums are long enough to be shared out."""
    out, p, want, z, bar, pre_bar = check_linear(aa, dtype, m, k, n, "silu", True, True, True)
    close(out, want, bar)
    close(p, z, pre_bar)
    check_grad(aa, dtype, m, k, n, "silu", True)
    x, w = mat(m, k, 1, dtype), mat(n, k, 2, dtype, std=k ** -0.5)
    x[m // 2:] = float("nan")
    out = like((m, n), dtype)
    aa.aa_linear(x, w, out, count_dev=i32([m // 2]))
    want, z, size = S.linear(f64(x)[:m // 2], f64(w), None, None, None)
    close(out[:m // 2], want, c(k) * size + HALF[dtype] * np.abs(want))
    assert torch.all(out[m // 2:] == 7.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m", [1, 2, 7, 8, 9, 15, 16])
@pytest.mark.parametrize("k,n", [(512, 4000), (96, 33), (33, 17), (1000, 1030), (2049, 70), (8, 15), (4096, 16)])
def test_linear_of_few_rows(aa, dtype, m, k, n):
    out, p, want, z, bar, pre_bar = check_linear(aa, dtype, m, k, n, "gelu", True, True, True)
    close(out, want, bar)
    close(p, z, pre_bar)
    out, _, want, _, bar, _ = check_linear(aa, dtype, m, k, n, None, False, False, False, (1, 3, 5), 1)
    close(out, want, bar)
    x, w = mat(m, k, 1, dtype), mat(n, k, 2, dtype)
    x[m // 2:] = float("nan")
    out = like((m, n), dtype)
    aa.aa_linear(x, w, out, count_dev=i32([m // 2]))
    assert torch.all(torch.isfinite(out[:m // 2])) and torch.all(out[m // 2:] == 7.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k,n,pads,shift", [(700, 515, 1001, (0, 0, 0), 0), (300, 1000, 1100, (0, 0, 0), 0), (520, 777, 700, (3, 1, 5), 1), (1100, 512, 640, (0, 0, 0), 0), (130, 1001, 2051, (0, 0, 0), 0)])
def test_linear_gradients_of_operands_that_are_copied(aa, dtype, m, k, n, pads, shift):
    """Large enough for copies of the operands in scratch memory; counted rows, whose successors hold NaN."""
    for act, residual in (("gelu", True), (None, False)):
        check_grad(aa, dtype, m, k, n, act, residual, pads, shift)
    rows = m - 37
    x, w, dout = mat(m, k, 1, dtype, pads[0], shift), mat(n, k, 2, dtype, pads[1], shift), mat(m, n, 3, dtype, pads[2], shift)
    x[rows:] = float("nan")
    dout[rows:] = float("nan")
    dx, dw, db = like((m, k), dtype), like((n, k), dtype), torch.full((n,), 7.0, device=DEV)
    scratch = aa.linear_grad_scratch(x, w)
    scratch.fill_(255)                      # NaN in every type
    aa.aa_linear_grad(x, w, dout, scratch, dx=dx, dw=dw, dbias=db, count_dev=i32([rows]))
    got, size, _ = S.linear_grad(f64(x)[:rows], f64(w), f64(dout)[:rows], None, None, None)
    close(dx[:rows], got["dx"], c(n) * size["dx"] + HALF[dtype] * np.abs(got["dx"]))
    assert torch.all(dx[rows:] == 7.0)
    close(dw, got["dw"], c(rows) * size["dw"] + HALF[dtype] * np.abs(got["dw"]))
    close(db, got["dbias"], c(rows) * size["dbias"])
