"""Host-side refusals of linear layers, layer normalisation and AdamW that need no GPU: the calls end before anything is enqueued.  And the C structures."""
import ctypes
import glob
import os
import re
import subprocess

import pytest
import torch

from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build

# the descriptors below hold no real addresses, so no call may get as far as a device
no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="refusals are looked at where nothing can run")
F32, BF16 = B.AA_F32, B.AA_BF16
BAD, TOO_LARGE, SMALL = B.AA_ERR_INVALID_ARG, B.AA_ERR_UNSUPPORTED, B.AA_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.lib()


def mat(at, rows, cols, dtype=BF16, stride=None):
    return B.aa_rows(at << 30, dtype, 0, rows, cols, cols if stride is None else stride)


def linear(lib, x, w, out, bias=None, act=0, residual=None, offsets=None, n_seg=0, pre=None):
    p = [ctypes.byref(m) if m is not None else None for m in (x, w, residual, pre, out)]
    return lib.aa_linear(ctypes.create_string_buffer(1 << 16), p[0], p[1], bias, act, p[2], offsets, n_seg, None, p[3], p[4])


@no_device
def test_linear_refusals(lib):
    x, w, out = mat(1, 6, 16), mat(2, 8, 16), mat(3, 6, 8)
    assert linear(lib, mat(1, 0, 16), w, mat(3, 0, 8)) == B.AA_OK                  # no rows: nothing to enqueue
    assert linear(lib, x, w, out, act=4) == linear(lib, x, w, out, act=-1) == BAD
    assert linear(lib, None, w, out) == linear(lib, x, None, out) == linear(lib, x, w, None) == BAD
    assert linear(lib, x, w, out, n_seg=3) == linear(lib, x, w, out, offsets=1 << 20, n_seg=-1) == BAD
    assert linear(lib, x, w, out, bias=(5 << 30) + 2) == BAD
    assert linear(lib, x, mat(2, 8, 16, F32), out) == linear(lib, x, w, mat(3, 6, 8, F32)) == BAD
    assert linear(lib, x, mat(2, 8, 17), out) == linear(lib, x, w, mat(3, 6, 9)) == linear(lib, x, w, mat(3, 5, 8)) == BAD
    assert linear(lib, x, w, out, residual=mat(4, 6, 7)) == linear(lib, x, w, out, pre=mat(4, 7, 8)) == BAD
    assert linear(lib, mat(1, 6, 16, stride=15), w, out) == linear(lib, B.aa_rows((1 << 30) + 1, BF16, 0, 6, 16, 16), w, out) == BAD
    assert linear(lib, mat(1, 6, 16, 7), mat(2, 8, 16, 7), mat(3, 6, 8, 7)) == BAD
    # what is written lies in nothing else; out may be the residual, with its stride
    assert linear(lib, x, w, mat(1, 6, 8)) == linear(lib, x, w, mat(2, 6, 8)) == linear(lib, x, w, out, pre=out) == BAD
    assert linear(lib, x, w, out, residual=mat(3, 6, 8, stride=9)) == linear(lib, x, w, out, pre=mat(4, 6, 8), residual=mat(4, 6, 8)) == BAD
    assert linear(lib, x, w, out, bias=3 << 30) == BAD
    # widths and rows that do not fit
    assert linear(lib, mat(1, 6, (1 << 30) + 1), mat(9, 1, (1 << 30) + 1), mat(3, 6, 1)) == TOO_LARGE
    assert linear(lib, mat(1, 1 << 31, 1), mat(900, 1, 1), mat(999, 1 << 31, 1)) == TOO_LARGE


@no_device
def test_linear_gradient_refusals(lib):
    x, w, dout, dx, dw = mat(1, 6, 16), mat(2, 8, 16), mat(3, 6, 8), mat(4, 6, 16), mat(5, 8, 16)
    need = ctypes.c_size_t(0)
    assert lib.aa_linear_grad_scratch_bytes(ctypes.byref(x), ctypes.byref(w), 0, ctypes.byref(need)) == B.AA_OK and need.value > 0
    assert lib.aa_linear_grad_scratch_bytes(ctypes.byref(x), ctypes.byref(w), 9, ctypes.byref(need)) == BAD
    assert lib.aa_linear_grad_scratch_bytes(ctypes.byref(x), ctypes.byref(w), 0, None) == BAD
    lib.aa_linear_grad_scratch_bytes(ctypes.byref(x), ctypes.byref(w), 2, ctypes.byref(need))

    def grad(x=x, w=w, act=0, pre=None, dout=dout, residual=None, dx=dx, dw=dw, dbias=6 << 30, scratch=7 << 30, size=None):
        p = [ctypes.byref(m) if m is not None else None for m in (x, w, pre, dout, residual, dx, dw)]
        return lib.aa_linear_grad(ctypes.create_string_buffer(1 << 16), p[0], p[1], act, p[2], p[3], p[4], None, 0, None, p[5], p[6], dbias, scratch,
                                  need.value if size is None else size)

    assert grad(act=2) == grad(pre=mat(8, 6, 8)) == BAD                             # pre exactly where there is an activation
    assert grad(residual=mat(8, 6, 16), dx=None) == grad(residual=mat(8, 6, 15)) == BAD
    assert grad(dout=None) == grad(dout=mat(3, 6, 9)) == grad(dx=mat(4, 6, 8)) == grad(dw=mat(5, 8, 15)) == BAD
    for i in (1, 2, 3):
        assert grad(dx=mat(i, 6, 16)) == grad(dw=mat(i, 8, 16)) == grad(dbias=i << 30) == BAD
    assert grad(dx=mat(5, 6, 16)) == grad(dbias=4 << 30) == grad(dbias=5 << 30) == grad(dbias=(6 << 30) + 1) == BAD
    assert grad(scratch=None) == grad(scratch=(7 << 30) + 128) == BAD
    assert grad(size=0) == grad(size=need.value // 2) == SMALL


def test_linear_gradient_scratch_follows_the_operands(lib):
    """What no product of the sizes can use is not asked for; the largest layers ask for no more than three rounds of tiles or the sums' parts."""
    def need(rows, inner, cols, dtype=BF16, act=0):
        n = ctypes.c_size_t(0)
        x, w = mat(1, rows, inner, dtype), mat(900, cols, inner, dtype)
        assert lib.aa_linear_grad_scratch_bytes(ctypes.byref(x), ctypes.byref(w), act, ctypes.byref(n)) == B.AA_OK
        return n.value

    sums, tile = 148 * 4, 256 * 260 * 4
    assert need(1, 64, 64) <= 64 * sums + 256 and need(0, 8, 8) <= 8 * sums + 256
    assert need(128, 128, 384) <= 384 * sums + 256                                  # sums of up to seven slices of 64 are not cut
    assert need(512, 64, 64) <= 2 * tile + 256 and need(449, 64, 64) == need(512, 64, 64) > need(448, 64, 64)
    assert need(2000, 256, 256) <= 8 * tile + 256 and need(16384, 256, 256) <= 16 * tile + 256
    assert need(25000, 512, 32000) <= 3 * 74 * 256 * 256 * 4 + 256
    assert need(64, 64, 64, F32) <= 64 * sums + 256 + 3 * 6 * 64 * 64 and need(64, 64, 64, BF16, 1) <= 64 * sums + 256 + 2 * 64 * 64


@no_device
def test_layer_norm_refusals(lib):
    ctx = ctypes.create_string_buffer(1 << 16)
    r = ctypes.byref

    def norm(x, out, eps=1e-5, gamma=None, beta=None):
        return lib.aa_layer_norm(ctx, r(x), gamma, beta, eps, None, 0, None, r(out))

    x, y = mat(1, 6, 16), mat(2, 6, 16)
    assert norm(mat(1, 0, 16), mat(2, 0, 16)) == B.AA_OK
    assert norm(x, mat(2, 6, 15)) == norm(x, mat(2, 6, 16, F32)) == norm(x, y, -1.0) == norm(x, y, float("nan")) == BAD
    assert norm(x, y, gamma=(3 << 30) + 1) == norm(x, y, gamma=2 << 30) == norm(x, y, beta=2 << 30) == norm(x, mat(1, 6, 16, stride=17)) == BAD
    need = ctypes.c_size_t(0)
    lib.aa_layer_norm_grad_scratch_bytes(r(x), r(need))

    def grad(dout=y, dx=mat(3, 6, 16), residual=None, dgamma=4 << 30, dbeta=5 << 30, scratch=6 << 30, size=None, gamma=None):
        return lib.aa_layer_norm_grad(ctx, r(x), gamma, 1e-5, r(dout), None if residual is None else r(residual), None, 0, None, r(dx), dgamma, dbeta, scratch,
                                      need.value if size is None else size)

    assert need.value > 0 and grad(size=need.value - 1) == SMALL and grad(scratch=(6 << 30) + 8) == grad(scratch=None) == BAD
    assert grad(dout=mat(2, 5, 16)) == grad(dx=mat(3, 6, 17)) == grad(residual=mat(8, 6, 15)) == grad(dx=mat(2, 6, 16, stride=20)) == BAD
    assert grad(dgamma=5 << 30) == grad(dgamma=1 << 30) == grad(dbeta=2 << 30) == grad(dbeta=3 << 30) == grad(gamma=4 << 30) == grad(gamma=3 << 30) == BAD


@no_device
def test_adamw_refusals(lib):
    ctx = ctypes.create_string_buffer(1 << 16)

    def step(n=64, param=1 << 30, grad=2 << 30, m=3 << 30, v=4 << 30, ms=None, vs=None, copy=None, decay=0.0, dtype=F32, bits=32, **rule):
        t = (B.aa_adamw_tensor * 1)(B.aa_adamw_tensor(param, grad, m, v, ms, vs, copy, n, decay, dtype, bits))
        return lib.aa_adamw(ctx, t, 1, ctypes.byref(B.adamw_rule(**{"lr": 0.1, **rule})), None)

    assert step(n=0) == B.AA_OK
    assert step(n=-1) == step(dtype=3) == step(bits=16) == step(decay=float("nan")) == BAD
    assert step(param=None) == step(grad=None) == step(m=None) == step(v=None) == step(bits=8) == step(bits=8, ms=5 << 30) == BAD
    assert step(param=(1 << 30) + 2) == step(grad=(2 << 30) + 2) == step(dtype=BF16, grad=(2 << 30) + 1) == step(copy=(5 << 30) + 1) == step(m=(3 << 30) + 1) == BAD
    assert step(m=1 << 30) == step(v=(3 << 30) + 252) == step(grad=1 << 30) == step(copy=2 << 30) == step(bits=8, ms=5 << 30, vs=5 << 30) == BAD
    assert step(n=(1 << 33) + 1) == TOO_LARGE
    for bad in ({"lr": -0.1}, {"lr": float("inf")}, {"beta1": 1.0}, {"beta2": float("nan")}, {"eps": -1e-9}, {"t": -1}):
        assert step(**bad) == BAD
    assert lib.aa_adamw(ctx, None, 1, ctypes.byref(B.adamw_rule(0.1)), None) == lib.aa_adamw(ctx, None, -1, ctypes.byref(B.adamw_rule(0.1)), None) == BAD


def test_structures_match_the_header(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = ['#include <stddef.h>', '#include "autoassist.h"']
    for name in ("aa_adamw_tensor", "aa_adamw_rule"):
        s = getattr(B, name)
        lines.append(f'_Static_assert(sizeof({name}) == {ctypes.sizeof(s)}, "{name}");')
        lines += [f'_Static_assert(offsetof({name}, {f[0]}) == {getattr(s, f[0]).offset}, "{name}.{f[0]}");' for f in s._fields_]
    lines += [f'_Static_assert(AA_ACT_{k} == {getattr(B, "AA_ACT_" + k)}, "{k}");' for k in ("NONE", "RELU", "GELU", "SILU")]
    src = tmp_path / "t.c"
    src.write_text("\n".join(lines) + "\n")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(root, "include"), "-c", str(src), "-o", str(tmp_path / "t.o")])


def test_kernels_that_start_early_read_by_ordinary_loads():
    """As for the other Boss operators: what the launch before may still write is not read through the read-only path."""
    files = [f for k in ("linear*", "layer_norm*", "adamw*", "cta_pair*") for f in glob.glob(os.path.join(build.CSRC, k))]
    assert len(files) >= 11
    for path in files:
        for n, line in enumerate(open(path), 1):
            code = line.split("//")[0]
            assert not re.search(r"__ldg\(|\.nc\b|__restrict__", code), f"{os.path.basename(path)}:{n}: {line.strip()}"
