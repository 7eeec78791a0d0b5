"""ngc_linear_xent / ngc_linear_xent_bwd through the C ABI against the fp64 oracle.

Bounds, elementwise, with U = 2^-24 one fp32 rounding.  A logit is a sum of `width` exact products (bf16) or rounded ones (fp32) in some
order: off by at most (width + 2) U sum |x w|.  lse is off by the largest such error of its row, plus the roundings of the sum of
exponentials and of the logarithm.  g is formed in fp32 and, for bf16 operands, rounded once to bf16 as the operand of the two products
that follow (2^-8 of its value); those are sums of exact products in fp32, rounded once to the result's type."""
import numpy as np
import pytest
import torch

import oracle
import paper_1801_08058_amd as ng
from tokens_util import CODE, HALF, TYPE, U, Guarded, stream, values, workspace, zipf_ids

pytestmark = pytest.mark.gpu


def _inputs(dtype, rows, width, vocab, seed, dead=0.1):
    x = values(seed, 0, (rows, width), 1.0, dtype)
    w = values(seed, 1, (vocab, width), 1.5 / max(1.0, width ** 0.5), dtype)
    labels = zipf_ids(seed, rows, vocab, dead)
    return x, w, labels, values(seed, 2, (rows,), 1.0, "f32")


def _check(dtype, x, w, labels, dloss, offset=0, grads=(True, True)):
    rows, width = x.shape
    vocab = w.shape[0]
    code, half = CODE[dtype], HALF[dtype]
    xd, wd = Guarded(x.size, TYPE[dtype], offset, x), Guarded(w.size, TYPE[dtype], offset, w)
    ld, gd = Guarded(rows, torch.int64, 0, labels), Guarded(rows, torch.float32, offset, dloss)
    loss, lse = Guarded(rows, torch.float32, offset), Guarded(rows, torch.float32, offset)
    ws, behind = workspace(ng.ngc_linear_xent_workspace_bytes(code, rows, width, vocab))
    ng.ngc_linear_xent(code, rows, width, vocab, xd.t, wd.t, ld.t, loss.t, lse.t, ws, stream())
    torch.cuda.synchronize()
    assert loss.intact() and lse.intact() and bool((behind == 0xFF).all())
    x64, w64 = x.astype(np.float64), w.astype(np.float64)
    z = x64 @ w64.T
    dz = (width + 2) * U * (np.abs(x64) @ np.abs(w64).T)
    ref_loss, ref_lse = oracle.linear_xent(x, w, labels)
    # sum of exponentials: each within 2^-22 of its value and of its argument's rounding, at most vocab / 64 + 64 additions deep
    dl = dz.max(1) + (vocab / 64 + 64) * U + 2.0 ** -21 * (1 + np.abs(z).max(1) + np.abs(ref_lse))
    live = (labels >= 0) & (labels < vocab)
    assert (np.abs(lse.f64(rows) - ref_lse) <= dl).all(), (np.abs(lse.f64(rows) - ref_lse) - dl).max()
    assert (np.abs(loss.f64(rows) - ref_loss) <= 2 * dl).all()
    assert (loss.f64(rows)[~live] == 0).all()
    if not any(grads):
        return
    lse_in = ref_lse.astype(np.float32)
    lse.t.copy_(torch.from_numpy(lse_in))
    ws, behind = workspace(ng.ngc_linear_xent_workspace_bytes(code, rows, width, vocab, True))
    dxd, dwd = (Guarded(v.size, TYPE[dtype], offset) if want else None for v, want in zip((x, w), grads))
    ng.ngc_linear_xent_bwd(code, rows, width, vocab, xd.t, wd.t, ld.t, lse.t, gd.t, dxd and dxd.t, dwd and dwd.t, ws, stream())
    torch.cuda.synchronize()
    assert bool((behind == 0xFF).all())
    ref = oracle.linear_xent_bwd(x, w, labels, lse_in, dloss)
    p = np.exp(z - lse_in.astype(np.float64)[:, None]) * np.where(live, np.abs(dloss), 0.0)[:, None]
    g = p.copy()
    g[np.flatnonzero(live), labels[live]] -= np.abs(dloss.astype(np.float64))[live]
    g = np.abs(g)
    arg = dz + (2.0 ** -20 * (1 + np.abs(lse_in)) + 2.0 ** -20 * np.abs(z).max(1))[:, None]      # of the exponential
    dg = (half * g if dtype == "bf16" else 0) + p * arg + 4 * U * g
    # subnormal values may be taken for zero, where the exponential leaves them, where the weight is applied and in the products
    dg = dg + 2.0 ** -124 * max(1.0, float(np.abs(dloss).max()))
    for out, want, other, k, gg, dd in ((dxd, ref[0], np.abs(w64), vocab, g, dg), (dwd, ref[1], np.abs(x64), rows, g.T, dg.T)):
        if out is None:
            continue
        got = out.f64(*want.shape)
        tol = dd @ other + (k + 8) * U * (gg @ other) + half * np.abs(want) + 2.0 ** -126
        err = np.abs(got - want)
        assert (err <= tol * 1.01).all(), (err - tol).max()
        # as a whole: two roundings of half a step each (g's and the result's), so no more than 2^-7 of the norm for bf16; fp32 sums far inside
        # 1e-5.  On top of either the exponential's argument: a probability is off by as much, relative to it, as its logit is absolutely
        # (a logit of 300 lies on a grid of 3e-5 in fp32).
        if want.size > 64 and np.linalg.norm(want):
            assert np.linalg.norm(got - want) <= ((2.0 ** -7 if dtype == "bf16" else 1e-5) + arg.max()) * np.linalg.norm(want)
        assert out.intact()
    if dxd is not None:
        assert (dxd.f64(rows, width)[~live] == 0).all()


SIZES = [(1, 1, 1), (1, 8, 2), (2, 7, 3), (3, 33, 63), (5, 64, 64), (64, 64, 65), (65, 72, 257), (17, 130, 1000), (130, 32, 1003), (257, 96, 300), (128, 256, 1000),
         (33, 515, 777), (300, 40, 4099), (8, 512, 10007), (520, 264, 520), (1, 1024, 5000), (70, 1000, 1024), (129, 136, 2049)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width,vocab", SIZES)
def test_loss_and_gradients(dtype, rows, width, vocab):
    print(f"linear_xent {rows} {width} {vocab} {dtype}", flush=True)
    _check(dtype, *_inputs(dtype, rows, width, vocab, rows + 3 * width + vocab))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width,vocab", [(5, 64, 64), (65, 72, 257), (130, 32, 1003), (33, 515, 777), (260, 128, 520)])
def test_tensors_off_the_16_byte_grid(dtype, rows, width, vocab):
    print(f"linear_xent offset {rows} {width} {vocab} {dtype}", flush=True)
    _check(dtype, *_inputs(dtype, rows, width, vocab, 7 + rows), offset=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grads", [(True, False), (False, True)])
def test_one_gradient_alone(dtype, grads):
    _check(dtype, *_inputs(dtype, 90, 200, 1500, 21), grads=grads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["none_live", "one_label", "uniform_mean", "zero_weights", "tiny_weights", "huge_logits", "row_masked_by_minus_30000"])
def test_special_rows(dtype, kind):
    rows, width, vocab = 150, 88, 900
    x, w, labels, dloss = _inputs(dtype, rows, width, vocab, 31)
    if kind == "none_live":
        labels[:] = -100
    elif kind == "one_label":
        labels[:] = vocab - 1
    elif kind == "uniform_mean":
        dloss[:] = 1.0 / 145
    elif kind == "zero_weights":
        dloss[:] = 0.0
    elif kind == "tiny_weights":
        dloss *= 1e-30
    elif kind == "huge_logits":
        x *= 64                                      # exponentials overflow without the shift; one class takes all the mass
    else:
        w[:, 0] = np.where(np.arange(vocab) % 3 == 0, 0.0, -30000.0 / 4)     # two thirds of the vocabulary masked by a bias feature
        w = oracle.bf16_bits_to_f64(oracle.f32_to_bf16_bits_rne(w.astype(np.float32))).astype(np.float32) if dtype == "bf16" else w
        x[:, 0] = 4.0
        labels = np.where(labels >= 0, labels // 3 * 3, labels)
    print(f"linear_xent special {kind} {dtype}", flush=True)
    _check(dtype, x, w, labels, dloss)


# rows and products split over many workgroups
@pytest.mark.parametrize("dtype,rows,width,vocab", [("bf16", 1030, 64, 5003), ("bf16", 2, 2048, 32000), ("f32", 3, 512, 20011), ("bf16", 4200, 24, 333),
                                                    ("f32", 700, 100, 3000), ("bf16", 600, 640, 9000)])
def test_long_axes(dtype, rows, width, vocab):
    print(f"linear_xent long {rows} {width} {vocab} {dtype}", flush=True)
    _check(dtype, *_inputs(dtype, rows, width, vocab, 41 + rows))


def test_results_do_not_depend_on_timing():
    x, w, labels, dloss = _inputs("bf16", 300, 256, 6000, 51)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()
    xd, wd, ld, gd = dev(x, torch.bfloat16), dev(w, torch.bfloat16), dev(labels, torch.int64), dev(dloss, torch.float32)
    got = []
    for fill in (0, 255):
        ws = torch.full((max(ng.ngc_linear_xent_workspace_bytes(ng.NGC_BF16, 300, 256, 6000, b) for b in (0, 1)),), fill, dtype=torch.uint8, device="cuda")
        loss, lse = torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
        dx, dw = torch.empty_like(xd), torch.empty_like(wd)
        ng.ngc_linear_xent(ng.NGC_BF16, 300, 256, 6000, xd, wd, ld, loss, lse, ws, stream())
        ng.ngc_linear_xent_bwd(ng.NGC_BF16, 300, 256, 6000, xd, wd, ld, lse, gd, dx, dw, ws, stream())
        torch.cuda.synchronize()
        got.append((loss, lse, dx, dw))
    for a, b in zip(*got):
        assert torch.equal(a, b)


# every tile of the products at sizes that end inside it (the sizes alone would choose the smallest for most of them)
@pytest.mark.parametrize("edge", [64, 128, 256])
@pytest.mark.parametrize("dtype,rows,width,vocab", [("bf16", 1, 8, 2), ("bf16", 300, 96, 777), ("bf16", 257, 515, 1003), ("bf16", 640, 264, 5003), ("f32", 130, 72, 300),
                                                    ("f32", 257, 515, 1003), ("bf16", 1100, 160, 3001)])
def test_every_tile(monkeypatch, edge, dtype, rows, width, vocab):
    print(f"linear_xent edge {edge} {rows} {width} {vocab} {dtype}", flush=True)
    monkeypatch.setenv("NGC_XENT_TILE", str(edge))
    _check(dtype, *_inputs(dtype, rows, width, vocab, 61 + rows))


# few rows and classes, long rows: the product in parts and a workgroup per row
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width,vocab", [(1, 4096, 3), (128, 2048, 1000), (7, 3001, 257), (40, 1500, 4097), (1000, 2000, 5), (1025, 2000, 5)])
def test_few_tiles_with_long_rows(dtype, rows, width, vocab):
    print(f"linear_xent parts {rows} {width} {vocab} {dtype}", flush=True)
    _check(dtype, *_inputs(dtype, rows, width, vocab, 71 + rows))


# few rows whose weight has to be read where it is (fp32, or rows off the 16-byte grid) over many classes
@pytest.mark.parametrize("dtype,rows,width,vocab", [("f32", 1, 64, 8192), ("f32", 5, 860, 9001), ("f32", 16, 33, 20011), ("f32", 17, 100, 8199), ("f32", 33, 7, 8300),
                                                    ("f32", 64, 130, 8205), ("f32", 65, 130, 8205), ("bf16", 1, 1, 8192), ("bf16", 3, 515, 10007), ("bf16", 16, 1030, 8193),
                                                    ("bf16", 40, 67, 8221), ("bf16", 64, 129, 9000), ("f32", 2, 5, 8191)])
def test_few_rows_over_many_classes(dtype, rows, width, vocab):
    print(f"linear_xent few {rows} {width} {vocab} {dtype}", flush=True)
    _check(dtype, *_inputs(dtype, rows, width, vocab, 81 + rows))
    _check(dtype, *_inputs(dtype, rows, width, vocab, 82 + rows), offset=1)


# more rows than one workgroup looks at in a step for the largest weight
@pytest.mark.parametrize("dtype,rows,width,vocab", [("bf16", 8192, 16, 40), ("bf16", 8193, 24, 40), ("f32", 20001, 20, 33)])
def test_many_rows(dtype, rows, width, vocab):
    print(f"linear_xent many {rows} {width} {vocab} {dtype}", flush=True)
    x, w, labels, dloss = _inputs(dtype, rows, width, vocab, 91 + rows)
    labels[-1], dloss[-1] = vocab // 2, 50.0                 # the largest weight in the last row
    _check(dtype, x, w, labels, dloss)


@pytest.mark.parametrize("rows,vocab", [(60, 500), (600, 9000), (17000, 40)])
def test_weights_of_rows_that_do_not_count(rows, vocab):
    x, w, labels, dloss = _inputs("bf16", rows, 32, vocab, 95 + rows)
    labels[::7] = -1
    dead = (labels < 0) | (labels >= vocab)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()
    xd, wd, ld = dev(x, torch.bfloat16), dev(w, torch.bfloat16), dev(labels, torch.int64)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ws = torch.empty(max(ng.ngc_linear_xent_workspace_bytes(ng.NGC_BF16, rows, 32, vocab, b) for b in (0, 1)), dtype=torch.uint8, device="cuda")
    ng.ngc_linear_xent(ng.NGC_BF16, rows, 32, vocab, xd, wd, ld, loss, lse, ws, stream())
    got = []
    for weight in (0.0, 3e38):
        dx, dw = torch.empty_like(xd), torch.empty_like(wd)
        gd = dev(np.where(dead, np.float32(weight), dloss), torch.float32)
        ng.ngc_linear_xent_bwd(ng.NGC_BF16, rows, 32, vocab, xd, wd, ld, lse, gd, dx, dw, ws, stream())
        torch.cuda.synchronize()
        got.append((dx, dw))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert bool((got[0][0][torch.from_numpy(dead).cuda()] == 0).all())


# two groups of rows, and the sizes around the ends of the rules
@pytest.mark.parametrize("dtype,rows,width,vocab", [("f32", 128, 515, 8200), ("f32", 97, 64, 9001), ("f32", 129, 40, 8300), ("f32", 32, 31, 8192), ("f32", 24, 1025, 8201),
                                                    ("bf16", 32, 131, 8195), ("bf16", 33, 131, 8195), ("f32", 100, 3, 8193), ("bf16", 9, 2, 8211)])
def test_few_rows_in_groups(dtype, rows, width, vocab):
    print(f"linear_xent groups {rows} {width} {vocab} {dtype}", flush=True)
    _check(dtype, *_inputs(dtype, rows, width, vocab, 84 + rows))
    _check(dtype, *_inputs(dtype, rows, width, vocab, 85 + rows), offset=1)
