"""ngc_layer_norm / ngc_layer_norm_bwd through the C ABI against the fp64 oracle.

Bounds, elementwise, with U = 2^-24 one fp32 rounding and `depth` the most additions that an element passes through on its way into a row's
sum (a lane's own share, then a tree): a row sum is off by at most depth U sum|.|.  Every result is then an expression of a few fp32
operations, rounded once to its type (HALF)."""
import numpy as np
import pytest
import torch

import oracle
import paper_1801_08058_amd as ng
from tokens_util import CODE, HALF, TYPE, U, Guarded, stream, values, workspace

pytestmark = pytest.mark.gpu


def _depth(cols):
    return cols / 64 + 48


def _inputs(dtype, rows, cols, seed, mean=0.0, std=1.0):
    x = values(seed, 0, (rows, cols), std, dtype, mean)
    return x, values(seed, 1, (rows, cols), 1.0, dtype), values(seed, 2, (cols,), 0.5, "f32", 1.0), values(seed, 3, (cols,), 0.5, "f32")


def _forward(dtype, x, gamma, beta, eps=1e-5, offset=0, in_place=False, stats=True):
    rows, cols = x.shape
    xd = Guarded(x.size, TYPE[dtype], offset, x)
    yd = xd if in_place else Guarded(x.size, TYPE[dtype], offset)
    gd, bd = (None if v is None else Guarded(cols, torch.float32, 1, v) for v in (gamma, beta))
    md, rd = (Guarded(rows, torch.float32) if stats else None for _ in range(2))
    ng.ngc_layer_norm(CODE[dtype], rows, cols, eps, xd.t, gd and gd.t, bd and bd.t, yd.t, md and md.t, rd and rd.t, stream())
    torch.cuda.synchronize()
    y, mean, rstd = oracle.layer_norm(x, gamma, beta, float(np.float32(eps)))
    d, xa = _depth(cols), np.abs(x.astype(np.float64))
    dm = (d + 2) * U * xa.mean(1)
    centred = x - mean[:, None]
    # (x - mean)^2: the mean's error enters squared, the rounding of the difference twice; then the sum, the division, the root
    var = (centred ** 2).mean(1)
    drel = ((d + 8) * U * var + dm ** 2) * rstd ** 2 + 4 * U
    g = np.abs(gamma) if gamma is not None else np.ones(cols)
    b = np.abs(beta) if beta is not None else np.zeros(cols)
    tol = (np.abs(centred) * rstd[:, None] * (drel + 6 * U)[:, None] + (dm * rstd)[:, None]) * g + 2 * U * b + np.abs(y) * HALF[dtype]
    err = np.abs(yd.f64(rows, cols) - y)
    assert (err <= tol * 1.001).all(), (err - tol).max()
    assert yd.intact()
    if stats:
        assert (np.abs(md.f64(rows) - mean) <= dm * 1.001).all()
        assert (np.abs(rd.f64(rows) - rstd) <= rstd * drel * 1.001).all()
        assert md.intact() and rd.intact()


def _backward(dtype, x, dy, gamma, offset=0, in_place=False, weights=(True, True)):
    rows, cols = x.shape
    _, mean, rstd = oracle.layer_norm(x)
    mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
    xd, dyd = Guarded(x.size, TYPE[dtype], offset, x), Guarded(x.size, TYPE[dtype], offset, dy)
    dxd = dyd if in_place else Guarded(x.size, TYPE[dtype], offset)
    gd = None if gamma is None else Guarded(cols, torch.float32, 1, gamma)
    md, rd = Guarded(rows, torch.float32, 1, mean), Guarded(rows, torch.float32, 1, rstd)
    dg, db = (Guarded(cols, torch.float32, 1) if w else None for w in weights)
    ws, behind = workspace(ng.ngc_layer_norm_workspace_bytes(CODE[dtype], rows, cols)) if any(weights) else (None, None)
    ng.ngc_layer_norm_bwd(CODE[dtype], rows, cols, xd.t, gd and gd.t, md.t, rd.t, dyd.t, dxd.t, dg and dg.t, db and db.t, ws, stream())
    torch.cuda.synchronize()
    dx, dgamma, dbeta = oracle.layer_norm_bwd(x, gamma, mean, rstd, dy)
    d, rs = _depth(cols), rstd.astype(np.float64)[:, None]
    xh = (x.astype(np.float64) - mean.astype(np.float64)[:, None]) * rs
    g = np.abs(dy if gamma is None else dy.astype(np.float64) * gamma)
    a, b = g.mean(1, keepdims=True), (g * np.abs(xh)).mean(1, keepdims=True)
    tol = rs * ((d + 6) * U * (a + np.abs(xh) * b) + 8 * U * (g + a + np.abs(xh) * b)) + np.abs(dx) * HALF[dtype]
    err = np.abs(dxd.f64(rows, cols) - dx)
    assert (err <= tol * 1.001).all(), (err - tol).max()
    assert dxd.intact()
    if weights[0]:
        assert (np.abs(dg.f64(cols) - dgamma) <= (rows + 5) * U * (np.abs(dy) * np.abs(xh)).sum(0) * 1.001).all() and dg.intact()
    if weights[1]:
        assert (np.abs(db.f64(cols) - dbeta) <= (rows + 5) * U * np.abs(dy.astype(np.float64)).sum(0) * 1.001).all() and db.intact()
    assert behind is None or bool((behind == 0xFF).all())


SIZES = [(1, 1), (2, 3), (5, 7), (3, 8), (4, 9), (70, 64), (33, 65), (9, 127), (17, 256), (300, 100), (6, 511), (5, 1000), (5, 1001), (3, 2048), (3, 2049),
         (260, 1024), (3, 4096), (2, 5000), (2, 8192), (2, 8200), (2, 12288), (3, 16384), (2, 16385), (2, 20001), (2, 32768), (2, 40000), (1, 65537)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(dtype, rows, cols):
    print(f"layer_norm {rows} {cols} {dtype}", flush=True)
    x, _, gamma, beta = _inputs(dtype, rows, cols, 100 + rows + cols)
    _forward(dtype, x, gamma, beta)
    _forward(dtype, x, gamma, None, offset=1, in_place=True)
    _forward(dtype, x, None, beta, eps=0.1, stats=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(dtype, rows, cols):
    print(f"layer_norm_bwd {rows} {cols} {dtype}", flush=True)
    x, dy, gamma, _ = _inputs(dtype, rows, cols, 200 + rows + cols)
    _backward(dtype, x, dy, gamma)
    _backward(dtype, x, dy, None, offset=1, in_place=True)
    _backward(dtype, x, dy, gamma, weights=(False, False))
    _backward(dtype, x, dy, gamma, weights=(True, False))
    _backward(dtype, x, dy, gamma, weights=(False, True))


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 5003, 96), ("f32", 3001, 33), ("bf16", 2100, 1032), ("bf16", 40000, 8), ("f32", 70000, 3), ("bf16", 1500, 16400)])
def test_many_rows(dtype, rows, cols):
    print(f"layer_norm many rows {rows} {cols} {dtype}", flush=True)
    x, dy, gamma, beta = _inputs(dtype, rows, cols, 300 + rows + cols)
    _forward(dtype, x, gamma, beta)
    _backward(dtype, x, dy, gamma)


@pytest.mark.parametrize("cols", [5, 100, 1000, 4096, 17000, 40000])
def test_rows_far_from_zero(cols):
    """The variance of values whose mean is a thousand times their spread: a difference of squares would lose it."""
    x, dy, gamma, beta = _inputs("f32", 4, cols, 400 + cols, mean=1000.0)
    x[1] -= 2000.0
    x[2] *= 1e3
    _forward("f32", x, gamma, beta)
    _backward("f32", x, dy, gamma)


def test_constant_rows_give_beta():
    x = np.repeat(np.array([[0.0], [3.0], [-1e4]], np.float32), 515, 1)
    _, _, gamma, beta = _inputs("f32", 3, 515, 5)
    _forward("f32", x, gamma, beta)
