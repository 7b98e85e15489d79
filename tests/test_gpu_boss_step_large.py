"""Linear layers and layer normalisation at sizes that fill the GPU - tiles of pairs of CTAs, several of them one after the other, contractions cut or summed in runs,
several rows a group of threads - against fp64 on the GPU.  Bars as in test_gpu_boss_step, and for the longest sums:
  bf16 sums: the matrix units round towards zero once in 16 terms, by half a step on average (2^-24 of the sum so far, which is half of the run's on average); runs of
             2,048 terms are added up in fp32.  So 128 2^-24 / 2 = 2^-18 of the sum of absolute terms, and 2^-24 of it for each run.
"""
import pytest
import torch

from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build
from test_gpu_boss_step import BF16, DEV, F32, HALF, c, i32
from test_gpu_boss_step_use import Layer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aa():
    build.build()
    ctx = B.AutoAssist(max_rows=1 << 10, max_d=64, device=DEV)
    yield ctx
    torch.cuda.synchronize()
    assert ctx.aa_device_status() == B.AA_OK
    ctx.close()


def random(shape, seed, dtype=BF16, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)


def below(got, bar):
    off = got.double().abs() - bar
    assert torch.all(off <= 0), f"off by {got.double().abs().max():.3e}, {off.max():.3e} above the bar"


def close(got, want, bar):
    assert torch.all(torch.isfinite(got))
    below(got.double() - want, bar)


def cancelling(rows, cols, seed, minus):
    """Numbers of [1, 2), then the same again (minus: with their signs turned)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    half = (1.0 + torch.rand((rows // 2, cols), generator=g, device=DEV)).to(BF16)
    return torch.cat([half, -half if minus else half])


def test_weights_gradients_of_many_tokens_keep_their_sums(aa):
    """Sums over 196,608 tokens whose second half takes back the first: every output is 0, and what it is off by has nowhere to hide."""
    tokens, n = 196_608, 2304                                     # 81 tiles of a pair: whole ones, and some that are cut
    x, dout = cancelling(tokens, n, 1, False), cancelling(tokens, n, 2, True)
    w = torch.zeros((n, n), dtype=BF16, device=DEV)
    dw, db = torch.empty_like(w), torch.empty(n, device=DEV)
    aa.aa_linear_grad(x, w, dout, aa.linear_grad_scratch(x, w), dw=dw, dbias=db)
    half = tokens // 2
    size = 2.0 * (x[:half].float().t() @ dout[:half].float()).t().double()
    below(dw, (2.0**-18 + tokens / 2048 * 2.0**-24) * size)
    # dbias: eight tokens at a time in fp32, rounded to nearest, of which a thread has every 32nd token
    below(db, tokens / 8 * 2.0**-24 * 2.0 * dout[:half].double().sum(0))


def test_long_contractions_keep_their_sums(aa):
    """The same along the inputs of a layer, forward and in dx."""
    k = 131_072
    x = cancelling(k, 2048, 3, True).t().contiguous()
    w = cancelling(k, 1100, 4, False).t().contiguous()
    out = torch.empty((2048, 1100), dtype=BF16, device=DEV)
    aa.aa_linear(x, w, out)
    size = 2.0 * (x[:, :k // 2].float() @ w[:, :k // 2].float().t()).double()
    below(out, (2.0**-18 + k / 2048 * 2.0**-24) * size)
    dout, w = cancelling(k, 1100, 5, True).t().contiguous(), cancelling(k, 2048, 6, False)
    x = torch.zeros((1100, 2048), dtype=BF16, device=DEV)
    dx = torch.empty_like(x)
    aa.aa_linear_grad(x, w, dout, aa.linear_grad_scratch(x, w), dx=dx)
    size = 2.0 * (dout[:, :k // 2].float() @ w[:k // 2].float()).double()
    below(dx, (2.0**-18 + k / 2048 * 2.0**-24) * size)


ACT = {None: lambda z: z, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}


# the first two of each: 54 and 153 tiles for 74 pairs of CTAs; the odd one has rows whose ends no vector meets
@pytest.mark.parametrize("dtype,m,k,n", [(BF16, 1300, 72, 2056), (BF16, 2100, 264, 4104), (BF16, 1111, 520, 4101), (F32, 1300, 65, 2051)])
@pytest.mark.parametrize("act", [None, "gelu", "relu"])
def test_linear_on_tiles_of_pairs(aa, dtype, m, k, n, act):
    x, w, bias = random((m, k), 1, dtype), random((n, k), 2, dtype, k ** -0.5), random((n,), 3, F32, 0.5)
    res = random((m, n), 4, dtype)
    out, pre = torch.empty_like(res), torch.empty_like(res)
    for rows in (m, m - 77, 257, 1):
        x[rows:] = float("nan")
        res[rows:] = float("nan")
        out.fill_(7.0), pre.fill_(7.0)
        aa.aa_linear(x, w, out, bias=bias, activation=act, residual=res, pre=pre, count_dev=i32([rows]))
        X, W = x[:rows].double(), w.double()
        z = X @ W.t() + bias.double()
        size = X.abs() @ W.t().abs() + bias.double().abs()
        want = ACT[act](z) + res[:rows].double()
        close(pre[:rows], z, c(k) * size + HALF[dtype] * z.abs())
        close(out[:rows], want, 1.13 * c(k) * size + 2.0**-20 * z.abs().clamp(min=1.0) * (act is not None) + HALF[dtype] * want.abs() + 2.0**-22 * z.abs())
        assert torch.all(out[rows:] == 7.0) and torch.all(pre[rows:] == 7.0)


def check_grad(aa, dtype, m, k, n, act, counts, which=("dx", "dw", "dbias")):
    """Counted rows have NaN behind them; counts are taken from the largest on."""
    x, w, dout = random((m, k), 1, dtype), random((n, k), 2, dtype, k ** -0.5), random((m, n), 3, dtype)
    pre, res = random((m, n), 4, dtype) if act else None, random((m, k), 5, dtype)
    z = None if pre is None else pre.double().requires_grad_()
    G = dout.double() if act is None else torch.autograd.grad(ACT[act](z), z, dout.double())[0]
    absolute = 2.0**-20 * (act not in (None, "relu"))              # of a slope
    rounded = 2.0**-8 if dtype == BF16 and act not in (None, "relu") else 0.0
    scratch = aa.linear_grad_scratch(x, w, act)
    for rows in counts:
        for t in (x, dout, res) + (() if pre is None else (pre,)):
            t[rows:] = float("nan")
        scratch.fill_(255)                                        # NaN in every type
        got = {"dx": torch.full_like(x, 7.0), "dw": torch.full_like(w, 7.0), "dbias": torch.full((n,), 7.0, device=DEV)}
        got = {name: got[name] for name in which}
        aa.aa_linear_grad(x, w, dout, scratch, activation=act, pre=pre, residual=res if "dx" in which else None, count_dev=i32([rows]), **got)
        X, W, g, d = x[:rows].double(), w.double(), G[:rows], dout[:rows].double().abs()
        if "dx" in which:
            want = g @ W + res[:rows].double()
            close(got["dx"][:rows], want, (c(n) + rounded) * (g.abs() @ W.abs()) + absolute * (d @ W.abs()) + (HALF[dtype] + 2.0**-22) * want.abs())
            assert torch.all(got["dx"][rows:] == 7.0)
        if "dw" in which:
            want = g.t() @ X
            close(got["dw"], want, (c(rows) + rounded) * (g.t().abs() @ X.abs()) + absolute * (d.t() @ X.abs()) + (HALF[dtype] + 2.0**-22) * want.abs())
        if "dbias" in which:
            close(got["dbias"], g.sum(0), c(rows) * g.abs().sum(0) + absolute * d.sum(0))


@pytest.mark.parametrize("act", [None, "relu", "silu"])
@pytest.mark.parametrize("m,k,n", [(5003, 520, 4616), (9001, 2312, 2320), (4999, 1000, 264)])
def test_gradients_on_tiles_of_pairs(aa, m, k, n, act):
    """Tiles of pairs in dx and dw: fewer than there are pairs, all of them cut; more, some of them cut; widths off the tiles.  Counts that end inside a slice of 64 tokens, at its
    end, and that leave nothing."""
    check_grad(aa, BF16, m, k, n, act, (m, m - 29, 4100, 128, 65, 64, 1, 0))


@pytest.mark.parametrize("act", [None, "gelu"])
def test_gradients_alone_on_tiles_of_pairs(aa, act):
    for which in (("dx",), ("dw",), ("dbias",), ("dw", "dbias"), ("dx", "dw")):
        check_grad(aa, BF16, 5003, 520, 4616, act, (4999,), which)


@pytest.mark.parametrize("m,k,n", [(3000, 2312, 17000), (17001, 600, 2312), (33000, 264, 640), (300_000, 264, 640)])
def test_gradients_whose_contractions_take_several_runs(aa, m, k, n):
    """Runs of whole tiles and of cut ones, with the sums of dout beside them."""
    check_grad(aa, BF16, m, k, n, None, (m, m - 29))


@pytest.mark.parametrize("act", [None, "silu"])
@pytest.mark.parametrize("m,k,n", [(2050, 1300, 2400), (2051, 1301, 2403)])
def test_fp32_gradients_with_several_tiles_a_pair(aa, m, k, n, act):
    check_grad(aa, F32, m, k, n, act, (m, m - 29, 65, 0))


def test_replayed_and_in_two_contexts_on_tiles_of_pairs():
    """Two layers of pairs' tiles, each captured on a stream of its own, replayed at once with other counts than at capture: the bits of calls alone and outside of graphs."""
    layers = []
    for m, k, n in ((5003, 520, 4616), (3000, 2312, 4104)):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            ctx = B.AutoAssist(max_rows=64, max_d=64, device=DEV, stream=stream)
            layer = Layer(ctx, BF16, m, k, n)
            layer.run()
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                layer.run()
        layers.append((stream, ctx, layer, graph, m))
    torch.cuda.synchronize()

    def fresh(layer, rows):
        layer.count.fill_(rows)
        for t in (layer.p, layer.m, layer.v):
            t.zero_()

    for less in (0, 29, 2900):
        alone = []
        for stream, _, layer, _, m in layers:
            with torch.cuda.stream(stream):
                fresh(layer, m - less)
                layer.run()
                alone.append(layer.results())
            torch.cuda.synchronize()
        for _ in range(3):
            for stream, _, layer, graph, m in layers:
                with torch.cuda.stream(stream):
                    fresh(layer, m - less)
                    graph.replay()
        torch.cuda.synchronize()
        for (stream, ctx, layer, _, _), want in zip(layers, alone):
            with torch.cuda.stream(stream):
                assert all(torch.equal(a, b) for a, b in zip(layer.results(), want))
                layer.check()
            assert ctx.aa_device_status() == B.AA_OK
    for _, ctx, _, _, _ in layers:
        ctx.close()


# ---------------------------------------------------------------------------------------------------------------------- norm

def norm_reference(x, gamma, eps):
    c = x - x.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    h = c * r
    return h, r, 2.0**-18 * (1.0 + h.abs()) + r * 2.0**-18 * x.abs().mean(1, keepdim=True)       # the last: what h may be off by


def strided(m, n, seed, dtype, pad):
    return random((m, n + pad), seed, dtype)[:, :n]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,pad", [(701, 4096, 0), (701, 4099, 0), (450, 5000, 0), (450, 5000, 3), (700, 8192, 0), (700, 8192, 1), (6001, 512, 0), (6001, 512, 5), (3001, 1024, 0), (2003, 2048, 0),
                                     (20001, 64, 0), (20001, 100, 0), (1201, 3000, 1), (40, 8200, 0), (300, 4609, 0), (300, 5203, 0), (300, 6101, 0), (300, 6145, 0), (300, 7001, 0), (300, 7603, 0), (300, 6144, 0), (300, 6148, 0)])
def test_norm_with_several_rows_a_group(aa, dtype, m, n, pad):
    """More rows than the threads that are resident take at once; counts that leave an odd number of them to the last, with NaN behind; in place."""
    x, d, res = (strided(m, n, seed, dtype, pad) for seed in (1, 2, 3))
    x.mul_(1.5).add_(0.3)
    gamma, beta = 1.0 + random((n,), 4, F32, 0.3), random((n,), 5, F32, 0.3)
    scratch = aa.layer_norm_grad_scratch(x)
    for rows in (m, m - 1, m // 2 + 1, 3):
        for t in (x, d, res):
            t[rows:] = float("nan")
        live = {"count_dev": i32([rows])}
        X, D = x[:rows].double(), d[:rows].double()
        h, r, e = norm_reference(X, gamma, 1e-5)
        g = D * gamma.double()
        want = h * gamma.double() + beta.double()
        out = torch.full_like(x, 7.0)
        aa.aa_layer_norm(x, out, gamma=gamma, beta=beta, **live)
        close(out[:rows], want, gamma.double().abs() * e + (HALF[dtype] + 2.0**-22) * want.abs())
        assert torch.all(out[rows:] == 7.0)
        mg, mgh = g.abs().mean(1, keepdim=True), (g * h).abs().mean(1, keepdim=True)
        plain = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        bar = r * (2.0**-18 * (g.abs() + mg) + e * (mgh + mg) + h.abs() * ((g.abs() * e).mean(1, keepdim=True) + 2.0**-18 * mgh)) + 2.0**-17 * plain.abs()
        for residual, onto in ((None, None), (res, None), (res, d), (None, x)):
            dx = torch.full_like(x, 7.0) if onto is None else onto.clone()
            a, b = (dx if onto is x else x), (dx if onto is d else d)
            dg, db = torch.full((n,), 7.0, device=DEV), torch.full((n,), 7.0, device=DEV)
            behind = dx[rows:].clone()
            aa.aa_layer_norm_grad(a, b, dx, scratch, gamma=gamma, residual=residual, dgamma=dg, dbeta=db, **live)
            want = plain + (0.0 if residual is None else res[:rows].double())
            close(dx[:rows], want, bar + 2.0**-22 * want.abs() + HALF[dtype] * want.abs())
            assert torch.equal(dx[rows:].view(torch.int32 if dtype == F32 else torch.int16), behind.view(torch.int32 if dtype == F32 else torch.int16))
            close(dg, (D * h).sum(0), (D.abs() * e).sum(0) + c(rows) * (D * h).abs().sum(0))
            close(db, D.sum(0), c(rows) * D.abs().sum(0))


def far_bars(x, h, r):
    """What h may be off by where the mean is corrected: the first one is off by 2^-18 mean|x| (test_gpu_boss_step), its correction by 2^-18 of that; sums and quotients 2^-18."""
    return r * 2.0**-36 * x.abs().mean(1, keepdim=True) + 2.0**-18 * h.abs() + 2.0**-22


@pytest.mark.parametrize("n", [5, 100, 512, 515, 1024, 2047, 4096, 4099, 5000, 8191, 9000])
@pytest.mark.parametrize("value,eps", [(0.1, 1e-10), (1000.1, 1e-5), (-333.3, 1e-6)])
def test_norm_of_constant_fp32_rows(aa, n, value, eps):
    """h is 0, whatever the rounding of a sum of n equal numbers."""
    m = 7
    x, d = torch.full((m, n), value, device=DEV), random((m, n), 2, F32)
    beta = random((n,), 3, F32)
    out, dx, dg, db = torch.empty_like(x), torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    aa.aa_layer_norm(x, out, beta=beta, eps=eps)
    r, h = eps**-0.5, torch.zeros((m, n), dtype=torch.float64, device=DEV)
    e = far_bars(x.double(), h, r)
    close(out, beta.double().expand(m, n), e + 2.0**-24 * beta.double().abs())
    aa.aa_layer_norm_grad(x, d, dx, aa.layer_norm_grad_scratch(x), eps=eps, dgamma=dg, dbeta=db)
    g = d.double()
    want = r * (g - g.mean(1, keepdim=True))
    # the variance that is left is 2^-18 of the square of the first mean's error: (2^-18 x)^2 2^-18 / eps of r at most
    close(dx, want, r * 2.0**-18 * (g.abs() + g.abs().mean(1, keepdim=True)) + want.abs() * (2.0**-18 * (2.0**-18 * value) ** 2 / eps + 2.0**-20) + r * 4.0 * e)
    close(dg, torch.zeros(n, dtype=torch.float64, device=DEV), (g.abs() * e).sum(0))


@pytest.mark.parametrize("m,n,pad", [(40, 64, 0), (40, 512, 0), (40, 515, 0), (700, 1024, 0), (701, 4096, 0), (701, 4099, 0), (30, 6000, 1), (12, 9000, 0)])
def test_norm_of_fp32_rows_far_from_zero(aa, m, n, pad):
    x, d = strided(m, n, 1, F32, pad), strided(m, n, 2, F32, pad)
    x.add_(1.0e4)
    gamma = 1.0 + random((n,), 4, F32, 0.3)
    h, r, _ = norm_reference(x.double(), gamma, 1e-5)
    e = far_bars(x.double(), h, r)
    out = torch.empty_like(x)
    aa.aa_layer_norm(x, out, gamma=gamma)
    close(out, h * gamma.double(), gamma.double().abs() * e + 2.0**-22 * h.abs())
    dx, dg = torch.empty_like(x), torch.empty(n, device=DEV)
    aa.aa_layer_norm_grad(x, d, dx, aa.layer_norm_grad_scratch(x), gamma=gamma, dgamma=dg)
    D = d.double()
    g = D * gamma.double()
    mg, mgh = g.abs().mean(1, keepdim=True), (g * h).abs().mean(1, keepdim=True)
    want = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    close(dx, want, r * (2.0**-18 * (g.abs() + mg) + e * (mgh + mg) + h.abs() * ((g.abs() * e).mean(1, keepdim=True) + 2.0**-18 * mgh)) + 2.0**-17 * want.abs())
    close(dg, (D * h).sum(0), (D.abs() * e).sum(0) + c(m) * (D * h).abs().sum(0))


# --------------------------------------------------------------------------------------------------------------- activations

@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_fp32_activations_and_slopes_number_by_number(aa, act):
    """One weight of 1 and one term a sum, so that the call gives act(z) itself, and dbias of one row act'(z).  erfc and exp are good to 2^-21; their arguments, rounded twice, move
    them by z^2 2^-23 of themselves."""
    z = torch.cat([torch.linspace(-12.0, 12.0, 100_001, device=DEV), torch.linspace(-2.0, 2.0, 50_000, device=DEV)])
    one, n = torch.ones((1, 1), device=DEV), z.numel()
    Z = z.double()
    e = 2.0**-21 + Z * Z * 2.0**-23
    if act == "gelu":
        q, phi = 0.5 * torch.special.erfc(Z.abs() * 0.5**0.5), torch.exp(-0.5 * Z * Z) * (0.5 / torch.pi) ** 0.5
        cdf = torch.where(Z > 0, 1.0 - q, q)
        want, slope = Z * cdf, cdf + Z * phi
        bar, slope_bar = Z.abs() * (q * e + 2.0**-24 * (Z > 0)) + 2.0**-23 * want.abs(), q * e + Z.abs() * phi * e + 2.0**-23 * cdf
    else:
        s = torch.sigmoid(Z)
        want, slope = Z * s, s * (1.0 + Z * (1.0 - s))
        bar, slope_bar = want.abs() * 2.0**-20, s * (1.0 + Z.abs()) * 2.0**-22
    for rows in (n, 12):                                          # tiles, and few rows
        x, out = z[:rows, None].contiguous(), torch.empty((rows, 1), device=DEV)
        aa.aa_linear(x, one, out, activation=act)
        close(out[:, 0], want[:rows], bar[:rows])
    w, pre, dout, db = torch.ones((n, 1), device=DEV), z[None, :].contiguous(), torch.ones((1, n), device=DEV), torch.empty(n, device=DEV)
    aa.aa_linear_grad(one, w, dout, aa.linear_grad_scratch(one, w, act), dbias=db, activation=act, pre=pre)
    close(db, slope, slope_bar)


# ------------------------------------------------------------------------------------------------------------------ surroundings

def padded(m, n, seed, dtype, pad, shift=0):
    """m x n with `shift` NaN before and `pad` NaN behind each row."""
    whole = torch.full((m, shift + n + pad), float("nan"), dtype=dtype, device=DEV)
    whole[:, shift:shift + n] = random((m, n), seed, dtype)
    return whole, whole[:, shift:shift + n]


def target(m, n, dtype, pad, shift=0):
    whole = torch.full((m, shift + n + pad), 7.0, dtype=dtype, device=DEV)
    return whole, whole[:, shift:shift + n]


def untouched(whole, n, shift):
    assert torch.all(whole[:, :shift] == 7.0) and torch.all(whole[:, shift + n:] == 7.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(8, 0), (16, 8), (3, 0), (5, 1), (0, 4)])
@pytest.mark.parametrize("m,k,n", [(9, 72, 40), (140, 72, 136), (700, 515, 1001), (1300, 264, 2056)])
def test_nothing_around_the_rows_is_read_into_them_or_written(aa, dtype, m, k, n, pad, shift):
    (_, x), (_, w), (_, dout), (_, pre), (_, res) = (padded(a, b, i, dtype, pad, shift) for i, (a, b) in enumerate(((m, k), (n, k), (m, n), (m, n), (m, n)), 1))
    w.mul_(k ** -0.5)
    (out_whole, out), (z_whole, z) = (target(m, n, dtype, pad, shift) for _ in range(2))
    aa.aa_linear(x, w, out, activation="relu", residual=res, pre=z)
    want = x.double() @ w.double().t()
    size = x.double().abs() @ w.double().t().abs()
    close(z, want, c(k) * size + HALF[dtype] * want.abs())
    want = want.clamp(min=0.0) + res.double()
    close(out, want, c(k) * size + (HALF[dtype] + 2.0**-22) * want.abs() + 2.0**-22 * size)
    untouched(out_whole, n, shift), untouched(z_whole, n, shift)
    for act in (None, "relu"):
        (dx_whole, dx), (dw_whole, dw) = target(m, k, dtype, pad, shift), target(n, k, dtype, pad, shift)
        db = torch.empty(n, device=DEV)
        aa.aa_linear_grad(x, w, dout, aa.linear_grad_scratch(x, w, act), dx=dx, dw=dw, dbias=db, activation=act, pre=pre if act else None)
        g = dout.double() * (1.0 if act is None else (pre > 0).double())
        for got, a, b, terms in ((dx, g, w.double(), n), (dw, g.t(), x.double(), m)):
            want = a @ b
            close(got, want, c(terms) * (a.abs() @ b.abs()) + (HALF[dtype] + 2.0**-22) * want.abs())
        close(db, g.sum(0), c(m) * g.abs().sum(0))
        untouched(dx_whole, k, shift), untouched(dw_whole, k, shift)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (5, 1), (0, 4)])
@pytest.mark.parametrize("m,n", [(9, 72), (700, 515), (300, 4099), (20, 9000)])
def test_nothing_around_normalised_rows_is_read_or_written(aa, dtype, m, n, pad, shift):
    (_, x), (_, d), (_, res) = (padded(m, n, i, dtype, pad, shift) for i in (1, 2, 3))
    (out_whole, out), (dx_whole, dx) = (target(m, n, dtype, pad, shift) for _ in range(2))
    dg, db = torch.full((n + 2,), 7.0, device=DEV), torch.full((n + 2,), 7.0, device=DEV)
    aa.aa_layer_norm(x, out)
    aa.aa_layer_norm_grad(x, d, dx, aa.layer_norm_grad_scratch(x), residual=res, dgamma=dg[1:-1], dbeta=db[1:-1])
    h, r, e = norm_reference(x.double(), None, 1e-5)
    close(out, h, e + HALF[dtype] * h.abs())
    D = d.double()
    mg, mgh = D.abs().mean(1, keepdim=True), (D * h).abs().mean(1, keepdim=True)
    plain = r * (D - D.mean(1, keepdim=True) - h * (D * h).mean(1, keepdim=True))
    want = plain + res.double()
    bar = r * (2.0**-18 * (D.abs() + mg) + e * (mgh + mg) + h.abs() * ((D.abs() * e).mean(1, keepdim=True) + 2.0**-18 * mgh)) + 2.0**-17 * plain.abs()
    close(dx, want, bar + 2.0**-22 * want.abs() + HALF[dtype] * want.abs())
    close(dg[1:-1], (D * h).sum(0), (D.abs() * e).sum(0) + c(m) * (D * h).abs().sum(0))
    close(db[1:-1], D.sum(0), c(m) * D.abs().sum(0))
    untouched(out_whole, n, shift), untouched(dx_whole, n, shift)
    assert all(v[0] == 7.0 and v[-1] == 7.0 for v in (dg, db))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_matrices_of_more_than_two_to_the_31_elements(aa, dtype):
    m, k, n = 70_001, 64, 32_000
    x, w, dout = random((m, k), 1, dtype), random((n, k), 2, dtype, 0.125), torch.empty((m, n), dtype=dtype, device=DEV)
    for i in range(0, m, 10_000):
        dout[i:i + 10_000] = random((min(10_000, m - i), n), 3 + i, dtype)
    out = torch.empty_like(dout)
    aa.aa_linear(x, w, out)
    rows = torch.tensor([0, 1, 2**31 // n - 1, 2**31 // n, 2**31 // n + 1, m - 300, m - 1], device=DEV)
    X, W = x[rows].double(), w.double()
    want = X @ W.t()
    close(out[rows], want, c(k) * (X.abs() @ W.t().abs()) + HALF[dtype] * want.abs())
    del out
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(n, device=DEV)
    aa.aa_linear_grad(x, w, dout, aa.linear_grad_scratch(x, w), dx=dx, dw=dw, dbias=db)
    g = dout[rows].double()
    want = g @ W
    close(dx[rows], want, c(n) * (g.abs() @ W.abs()) + (HALF[dtype] + 2.0**-22) * want.abs())
    cols = [0, 5, n // 2, n - 1]
    g = dout[:, cols].double()
    want = g.t() @ x.double()
    close(dw[cols], want, c(m) * (g.t().abs() @ x.double().abs()) + (HALF[dtype] + 2.0**-22) * want.abs())
    close(db[cols], g.sum(0), c(m) * g.abs().sum(0))
