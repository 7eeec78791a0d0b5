"""ngc_linear_xent / _bwd where a feature masks classes with the lowest number of the type: x[n][0] = 1 (or 4: the logit leaves the range of fp32)
and w[v][0] = lowest in the masked classes, 0 in the others.  A masked class has probability 0: loss and gradients are those of the other classes
alone, and a run of masked classes as long as a tile, or in front of all others, changes nothing.  Bounds as in test_gpu_linear_xent.py, of the
classes that are left."""
import numpy as np
import pytest
import torch

import oracle
import paper_1801_08058_amd as ng
from test_gpu_linear_xent import _inputs
from tokens_util import CODE, HALF, TYPE, U, Guarded, stream, workspace

pytestmark = pytest.mark.gpu

LOWEST = {"bf16": -float(torch.finfo(torch.bfloat16).max), "f32": -float(torch.finfo(torch.float32).max)}


def _run(dtype, x, w, labels, dloss):
    rows, width = x.shape
    vocab, code = w.shape[0], CODE[dtype]
    xd, wd = Guarded(x.size, TYPE[dtype], 0, x), Guarded(w.size, TYPE[dtype], 0, w)
    ld, gd = Guarded(rows, torch.int64, 0, labels), Guarded(rows, torch.float32, 0, dloss)
    loss, lse, dx, dw = Guarded(rows, torch.float32), Guarded(rows, torch.float32), Guarded(x.size, TYPE[dtype]), Guarded(w.size, TYPE[dtype])
    for bwd in (False, True):
        ws, behind = workspace(ng.ngc_linear_xent_workspace_bytes(code, rows, width, vocab, bwd))
        if bwd:
            ng.ngc_linear_xent_bwd(code, rows, width, vocab, xd.t, wd.t, ld.t, lse.t, gd.t, dx.t, dw.t, ws, stream())
        else:
            ng.ngc_linear_xent(code, rows, width, vocab, xd.t, wd.t, ld.t, loss.t, lse.t, ws, stream())
        torch.cuda.synchronize()
        assert bool((behind == 0xFF).all())
    assert all(t.intact() for t in (loss, lse, dx, dw))
    return loss.f64(rows), lse.f64(rows), dx.f64(rows, width), dw.f64(vocab, width)


def _masked(kind, vocab):
    v = np.arange(vocab)
    return {"behind": v >= vocab // 3, "in_front": v < vocab - vocab // 3, "every_other": v % 2 == 0, "all_but_one": v != vocab // 2}[kind]


# the logits in parts, in tiles of each size (rows above what the parts take, many rows), straight from memory (fp32, odd bf16 widths over many classes)
CASES = [("bf16", 5, 64, 900), ("bf16", 130, 72, 5003), ("bf16", 1100, 40, 3001), ("bf16", 3, 67, 9001), ("f32", 5, 64, 900), ("f32", 40, 33, 9001), ("f32", 1100, 40, 3001),
         ("bf16", 9000, 16, 300)]


@pytest.mark.parametrize("feature", [1.0, 4.0])
@pytest.mark.parametrize("kind", ["behind", "in_front", "every_other", "all_but_one"])
@pytest.mark.parametrize("dtype,rows,width,vocab", CASES)
def test_masked_classes_do_not_count(dtype, rows, width, vocab, kind, feature):
    print(f"linear_xent masked {kind} {feature} {rows} {width} {vocab} {dtype}", flush=True)
    x, w, labels, dloss = _inputs(dtype, rows, width, vocab, 17 + rows)
    masked = _masked(kind, vocab)
    kept = np.flatnonzero(~masked)
    x[:, 0], w[:, 0] = feature, np.where(masked, LOWEST[dtype], 0.0)
    live = (labels >= 0) & (labels < vocab)
    at = np.where(live, labels, 0) % kept.size
    labels = np.where(live, kept[at], labels)
    loss, lse, dx, dw = _run(dtype, x, w, labels, dloss)
    x64, left = x.astype(np.float64), w[kept].astype(np.float64)
    z = x64 @ left.T
    ref_loss, ref_lse = oracle.linear_xent(x, left, np.where(live, at, -1))
    arg = (width + 2) * U * (np.abs(x64) @ np.abs(left).T)
    dl = arg.max(1) + (vocab / 64 + 64) * U + 2.0 ** -21 * (1 + np.abs(z).max(1) + np.abs(ref_lse))
    assert (np.abs(lse - ref_lse) <= dl).all() and (np.abs(loss - ref_loss) <= 2 * dl).all()
    assert (loss[~live] == 0).all()
    ref = oracle.linear_xent_bwd(x, left, np.where(live, at, -1), lse, dloss)
    weight = np.where(live, np.abs(dloss.astype(np.float64)), 0.0)[:, None]
    p = np.exp(z - lse[:, None]) * weight
    g = p.copy()
    g[np.flatnonzero(live), at[live]] -= weight[live, 0]
    g = np.abs(g)
    arg = arg + (2.0 ** -20 * (1 + np.abs(lse)) + 2.0 ** -20 * np.abs(z).max(1))[:, None]
    dg = (HALF[dtype] * g if dtype == "bf16" else 0) + p * arg + 4 * U * g + 2.0 ** -124 * max(1.0, float(np.abs(dloss).max()))
    for got, want, other, k, gg, dd in ((dx, ref[0], np.abs(left), vocab, g, dg), (dw[kept], ref[1], np.abs(x64), rows, g.T, dg.T)):
        tol = dd @ other + (k + 8) * U * (gg @ other) + HALF[dtype] * np.abs(want) + 2.0 ** -126
        assert (np.abs(got - want) <= tol * 1.01).all(), (np.abs(got - want) - tol).max()
    assert (dw[masked] == 0).all() and (dx[~live] == 0).all()


@pytest.mark.parametrize("dtype,rows,width,vocab", CASES)
def test_rows_without_a_class_that_do_not_count(dtype, rows, width, vocab):
    """Rows that see every class masked and have no label: a finite lse, no loss, and nothing of them in the gradients."""
    print(f"linear_xent empty rows {rows} {width} {vocab} {dtype}", flush=True)
    x, w, labels, dloss = _inputs(dtype, rows, width, vocab, 23 + rows, dead=0.0)
    empty = np.arange(rows) % 3 == 1
    labels[empty] = -100
    x[:, 0], w[:, 0] = np.where(empty, 1.0, 0.0), LOWEST[dtype]
    loss, lse, dx, dw = _run(dtype, x, w, labels, dloss)
    assert (np.abs(lse[empty] / LOWEST[dtype] - 1) <= 4 * U).all()       # lowest + log(vocab) + the other features, all below its last bit
    assert (loss[empty] == 0).all() and (dx[empty] == 0).all()
    rest = np.flatnonzero(~empty)
    _, lse1, dx1, dw1 = _run(dtype, x[rest], w, labels[rest], dloss[rest])
    # The same rows alone, perhaps in another order of additions: a rounding of g and one of the result on either side, and 2^-16 for fp32 sums
    # and exponentials of a few hundred rows and a few thousand classes
    w64, x64 = np.abs(w[:, 1:].astype(np.float64)), np.abs(x[rest][:, 1:].astype(np.float64))
    p = np.exp(x[rest][:, 1:].astype(np.float64) @ w[:, 1:].astype(np.float64).T - lse1[:, None])
    mass = (p + (np.arange(vocab) == labels[rest][:, None])) * np.abs(dloss[rest].astype(np.float64))[:, None]
    bound = 4 * HALF[dtype] + 2.0 ** -16
    assert np.abs(lse[rest] - lse1).max() <= 2.0 ** -16 * (1 + np.abs(lse1).max())
    assert (np.abs(dw[:, 1:] - dw1[:, 1:]) <= bound * (mass.T @ x64) + 2.0 ** -120).all() and (dw[:, 0] == 0).all()
    # (dx of feature 0 is the sum of g, about 0, times the lowest number)
    assert (np.abs(dx[rest][:, 1:] - dx1[:, 1:]) <= bound * (mass @ w64) + 2.0 ** -120).all()
