"""The gradients of ngc_linear_xent_bwd for few rows of bf16, and for more where the products are small: g enters its products with 16 bits, so that
dx and dw are one rounding away from those of an exact g.  Elementwise bounds as in test_gpu_linear_xent.py, with g's rounding at two half steps of bf16 on top of each other,
2^-8 of its value times 2^-8, in the place of one."""
import numpy as np
import pytest
import torch

import oracle
import paper_1801_08058_amd as ng
from test_gpu_linear_xent import _inputs
from tokens_util import U, Guarded, stream, workspace

pytestmark = pytest.mark.gpu


def _gradients(x, w, labels, lse, dloss, offset):
    rows, width = x.shape
    vocab = w.shape[0]
    fill = lambda a, t: Guarded(a.size, t, offset if t.is_floating_point else 0, a)
    xd, wd, ld, sd, gd = (fill(a, t) for a, t in ((x, torch.bfloat16), (w, torch.bfloat16), (labels, torch.int64), (lse, torch.float32), (dloss, torch.float32)))
    dx, dw = Guarded(x.size, torch.bfloat16, offset), Guarded(w.size, torch.bfloat16, offset)
    ws, behind = workspace(ng.ngc_linear_xent_workspace_bytes(ng.NGC_BF16, rows, width, vocab, True))
    ng.ngc_linear_xent_bwd(ng.NGC_BF16, rows, width, vocab, xd.t, wd.t, ld.t, sd.t, gd.t, dx.t, dw.t, ws, stream())
    torch.cuda.synchronize()
    assert dx.intact() and dw.intact() and bool((behind == 0xFF).all())
    return dx.f64(rows, width), dw.f64(vocab, width)


def _check(rows, width, vocab, offset):
    x, w, labels, dloss = _inputs("bf16", rows, width, vocab, 7 * rows + width + vocab, dead=0.1 if rows > 4 else 0.0)
    x64, w64 = x.astype(np.float64), w.astype(np.float64)
    lse = oracle.linear_xent(x, w, labels)[1].astype(np.float32)
    z = x64 @ w64.T
    live = (labels >= 0) & (labels < vocab)
    weight = np.where(live, np.abs(dloss.astype(np.float64)), 0.0)[:, None]
    p = np.exp(z - lse.astype(np.float64)[:, None]) * weight
    g = p.copy()
    g[np.flatnonzero(live), labels[live]] -= weight[live, 0]
    g = np.abs(g)
    arg = (width + 2) * U * (np.abs(x64) @ np.abs(w64).T) + (2.0 ** -20 * (1 + np.abs(lse)) + 2.0 ** -20 * np.abs(z).max(1))[:, None]
    dg = 2.0 ** -16 * g + p * arg + 4 * U * g + 2.0 ** -124 * max(1.0, float(np.abs(dloss).max()))
    want = oracle.linear_xent_bwd(x, w, labels, lse, dloss)
    for got, ref, other, k, gg, dd in zip(_gradients(x, w, labels, lse, dloss, offset), want, (np.abs(w64), np.abs(x64)), (vocab, rows), (g, g.T), (dg, dg.T)):
        tol = dd @ other + (k + 8) * U * (gg @ other) + 2.0 ** -8 * np.abs(ref) + 2.0 ** -126
        err = np.abs(got - ref)
        assert (err <= tol * 1.01).all(), (err - tol).max()


# the logits in parts, in tiles (one row over 70001 classes of 256; 128 rows over 9000), straight from memory (odd widths over many classes)
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("rows,width,vocab", [(1, 8, 2), (1, 64, 300), (2, 515, 777), (17, 130, 1000), (128, 256, 1000), (1, 256, 70001), (100, 72, 9000), (128, 512, 9000),
                                              (300, 515, 777), (1000, 128, 500), (1030, 64, 5003), (8193, 24, 40), (5000, 33, 300), (129, 520, 2049), (1024, 1024, 2048),
                                              (1, 33, 8192), (16, 67, 8221), (17, 131, 8195), (32, 515, 10007), (33, 129, 8300), (128, 8, 33)])
def test_few_rows_keep_sixteen_bits_of_g(rows, width, vocab, offset):
    print(f"linear_xent bits {rows} {width} {vocab} offset {offset}", flush=True)
    _check(rows, width, vocab, offset)


@pytest.mark.parametrize("edge", [64, 128, 256])
@pytest.mark.parametrize("rows,width,vocab", [(1, 16, 70), (3, 515, 1003), (100, 72, 777), (128, 264, 2500), (65, 130, 129), (700, 72, 1003)])
def test_sixteen_bits_with_every_tile(monkeypatch, rows, width, vocab, edge):
    print(f"linear_xent bits edge {edge} {rows} {width} {vocab}", flush=True)
    monkeypatch.setenv("NGC_XENT_TILE", str(edge))
    _check(rows, width, vocab, 0)


# parts, tiles, weights straight from memory
@pytest.mark.parametrize("rows,width,vocab", [(128, 256, 1000), (17, 512, 9000), (5, 67, 9001), (2000, 64, 3000)])
def test_captured_calls_replay_bit_for_bit(rows, width, vocab):
    print(f"linear_xent bits graph {rows} {width} {vocab}", flush=True)
    need = max(ng.ngc_linear_xent_workspace_bytes(ng.NGC_BF16, rows, width, vocab, b) for b in (0, 1))
    new = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")
    x, w, dx, dw, labels, ws = new(rows, width), new(vocab, width), new(rows, width), new(vocab, width), new(rows, t=torch.int64), new(need, t=torch.uint8)
    loss, lse, dloss = (new(rows, t=torch.float32) for _ in range(3))
    outs = (loss, lse, dx, dw)

    def run(st):
        ng.ngc_linear_xent(ng.NGC_BF16, rows, width, vocab, x, w, labels, loss, lse, ws, st)
        ng.ngc_linear_xent_bwd(ng.NGC_BF16, rows, width, vocab, x, w, labels, lse, dloss, dx, dw, ws, st)

    def load(seed):
        for t, a in zip((x, w, labels, dloss), _inputs("bf16", rows, width, vocab, seed)):
            t.copy_(torch.from_numpy(np.ascontiguousarray(a)))

    load(1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        run(side.cuda_stream)                            # eager: one-time kernel attributes are set outside the capture
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run(torch.cuda.current_stream().cuda_stream)
    for seed in (2, 3, 4):
        load(seed)
        run(stream())
        torch.cuda.synchronize()
        eager = [t.clone() for t in outs]
        for t in outs:
            t.fill_(float("nan"))
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)), seed
