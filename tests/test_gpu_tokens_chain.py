"""The operators over tokens and a vocabulary as a model runs them: tokens -> embedding -> layer norm -> softmax cross entropy with the table as
the last layer's weight -> all gradients back to the table.  Against the fp64 oracle stage by stage (each stage on what the device handed it),
against differences of the whole loss, and captured into a HIP graph."""
import numpy as np
import pytest
import torch

import oracle
import paper_1801_08058_amd as ng
from tokens_util import CODE, HALF, TYPE, values, zipf_ids

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Step:
    """A training step on static buffers."""

    def __init__(self, dtype, rows, width, vocab):
        self.dtype, self.rows, self.width, self.vocab, self.code = dtype, rows, width, vocab, CODE[dtype]
        data = lambda *s: torch.zeros(s, dtype=TYPE[dtype], device="cuda")
        f32 = lambda *s: torch.zeros(s, device="cuda")
        self.table, self.h, self.y, self.dy, self.dh, self.dw = (data(vocab, width), data(rows, width), data(rows, width), data(rows, width),
                                                                 data(rows, width), data(vocab, width))
        self.gamma, self.beta, self.mean, self.rstd, self.dgamma, self.dbeta = f32(width), f32(width), f32(rows), f32(rows), f32(width), f32(width)
        self.ids, self.labels = (torch.zeros(rows, dtype=torch.int64, device="cuda") for _ in range(2))
        self.loss, self.lse, self.dloss, self.dtable = f32(rows), f32(rows), f32(rows), f32(vocab, width)
        ws = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        self.ws = ws(max(ng.ngc_embedding_workspace_bytes(rows, vocab, width), ng.ngc_layer_norm_workspace_bytes(self.code, rows, width),
                         *(ng.ngc_linear_xent_workspace_bytes(self.code, rows, width, vocab, b) for b in (0, 1))))

    def outputs(self):
        return {n: getattr(self, n) for n in ("h", "y", "mean", "rstd", "loss", "lse", "dy", "dw", "dh", "dgamma", "dbeta", "dtable")}

    def load(self, seed):
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a))
        self.table.copy_(t(values(seed, 0, (self.vocab, self.width), 0.3, self.dtype)))
        self.gamma.copy_(t(values(seed, 1, (self.width,), 0.2, "f32", 1.0)))
        self.beta.copy_(t(values(seed, 2, (self.width,), 0.2, "f32")))
        self.ids.copy_(t(zipf_ids(seed, self.rows, self.vocab)))
        self.labels.copy_(t(zipf_ids(seed + 1, self.rows, self.vocab)))
        self.dloss.fill_(1.0 / self.rows)

    def run(self, st):
        r, w, v, c = self.rows, self.width, self.vocab, self.code
        ng.ngc_embedding(c, r, v, w, 2.0, self.table, self.ids, self.h, st)
        ng.ngc_layer_norm(c, r, w, EPS, self.h, self.gamma, self.beta, self.y, self.mean, self.rstd, st)
        ng.ngc_linear_xent(c, r, w, v, self.y, self.table, self.labels, self.loss, self.lse, self.ws, st)
        ng.ngc_linear_xent_bwd(c, r, w, v, self.y, self.table, self.labels, self.lse, self.dloss, self.dy, self.dw, self.ws, st)
        ng.ngc_layer_norm_bwd(c, r, w, self.h, self.gamma, self.mean, self.rstd, self.dy, self.dh, self.dgamma, self.dbeta, self.ws, st)
        ng.ngc_embedding_bwd(c, r, v, w, 2.0, self.dh, self.ids, self.dtable, self.ws, st)

    def f64(self, name):
        return getattr(self, name).double().cpu().numpy() if getattr(self, name).is_floating_point() else getattr(self, name).cpu().numpy()


def _near(got, want, bound):
    assert np.linalg.norm(got - want) <= bound * np.linalg.norm(want), np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("dtype,rows,width,vocab", [("f32", 150, 72, 700), ("bf16", 150, 72, 700), ("bf16", 515, 260, 5003), ("f32", 33, 515, 1001)])
def test_a_training_step_stage_by_stage(dtype, rows, width, vocab):
    print(f"chain {dtype} {rows} {width} {vocab}", flush=True)
    s = Step(dtype, rows, width, vocab)
    s.load(71 + rows)
    s.run(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    d = {n: s.f64(n) for n in (*s.outputs(), "table", "gamma", "beta", "ids", "labels", "dloss")}
    # One rounding to the type (two where g is rounded before its product) on fp32 arithmetic whose own error, relative to the norm of a
    # stage's result, stays far below 2^-16 at these sizes (sums of at most 5003 terms, rows that are not nearly constant)
    one, two = HALF[dtype] + 2.0 ** -16, 2 * HALF[dtype] + 2.0 ** -16
    _near(d["h"], oracle.embedding(d["table"], d["ids"], 2.0), one)
    y, mean, rstd = oracle.layer_norm(d["h"], d["gamma"], d["beta"], EPS)
    _near(d["y"], y, one), _near(d["rstd"], rstd, 2.0 ** -16)
    loss, lse = oracle.linear_xent(d["y"], d["table"], d["labels"])
    _near(d["loss"], loss, 2.0 ** -16), _near(d["lse"], lse, 2.0 ** -16)
    dy, dw = oracle.linear_xent_bwd(d["y"], d["table"], d["labels"], d["lse"], d["dloss"])
    _near(d["dy"], dy, two), _near(d["dw"], dw, two)
    dh, dgamma, dbeta = oracle.layer_norm_bwd(d["h"], d["gamma"], d["mean"], d["rstd"], d["dy"])
    _near(d["dh"], dh, one), _near(d["dgamma"], dgamma, 2.0 ** -16), _near(d["dbeta"], dbeta, 2.0 ** -16)
    _near(d["dtable"], oracle.embedding_bwd(d["dh"], d["ids"], vocab, 2.0), 2.0 ** -16)


def test_the_gradient_of_the_table_is_the_derivative_of_the_loss():
    """Both uses of the table: <gradient, direction> against the central difference of the loss in fp64.  The difference is off by h^2 / 6 times the
    third derivative (h = 1e-4: below 1e-6 of the slope here), the gradient by fp32 roundings of a few stages: 1e-3 leaves room for both."""
    rows, width, vocab = 60, 40, 90
    s = Step("f32", rows, width, vocab)
    s.load(5)
    s.run(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    table, gamma, beta, ids, labels, w = (s.f64(n) for n in ("table", "gamma", "beta", "ids", "labels", "dloss"))

    def loss(t):
        y, _, _ = oracle.layer_norm(oracle.embedding(t, ids, 2.0), gamma, beta, EPS)
        return float((oracle.linear_xent(y, t, labels)[0] * w).sum())

    grad = s.f64("dw") + s.f64("dtable")
    for seed in range(4):
        v = np.random.default_rng(seed).normal(size=table.shape) + grad / np.abs(grad).max()
        slope = (loss(table + 1e-4 * v) - loss(table - 1e-4 * v)) / 2e-4
        scale = np.linalg.norm(grad) * np.linalg.norm(v)
        assert abs((grad * v).sum() - slope) <= 1e-3 * max(abs(slope), 1e-2 * scale)


@pytest.mark.parametrize("dtype,rows,width,vocab", [("bf16", 130, 72, 700), ("bf16", 700, 256, 9000), ("f32", 130, 33, 3001), ("bf16", 5000, 64, 300)])
def test_a_captured_step_replays_bit_for_bit(dtype, rows, width, vocab):
    print(f"graph {dtype} {rows} {width} {vocab}", flush=True)
    s = Step(dtype, rows, width, vocab)
    side = torch.cuda.Stream()
    s.load(1)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.run(side.cuda_stream)                          # eager: one-time kernel attributes are set outside the capture
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s.run(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for seed in (2, 3, 4):
        s.load(seed)
        s.run(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        eager = {n: t.clone() for n, t in s.outputs().items()}
        assert all(torch.isfinite(t).all() for t in eager.values())
        for t in s.outputs().values():
            t.fill_(float("nan"))
        s.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in s.outputs().items():
            assert torch.equal(t, eager[n]), f"seed {seed}: {n}"


def test_two_steps_on_two_streams_do_not_touch_each_other():
    a, b = Step("bf16", 300, 128, 4000), Step("bf16", 257, 136, 5003)
    a.load(11), b.load(12)
    torch.cuda.synchronize()
    want = []
    for s in (a, b):
        s.run(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        want.append({n: t.clone() for n, t in s.outputs().items()})
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.run(sa.cuda_stream), b.run(sb.cuda_stream)
    torch.cuda.synchronize()
    for s, w in zip((a, b), want):
        for n, t in s.outputs().items():
            assert torch.equal(t, w[n]), n
