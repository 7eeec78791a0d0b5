"""ngc_linear_xent / _bwd over a vocabulary of several pieces: small ones, which NGC_XENT_PIECE cuts off a small vocabulary, against the fp64 oracle with the
bounds of test_gpu_linear_xent.py; and a size that has two by itself."""
import pytest
import torch

import paper_1801_08058_amd as ng
from test_gpu_linear_xent import _check, _inputs
from tokens_util import CODE, stream

pytestmark = pytest.mark.gpu


# last pieces of every kind (one class, no multiple of 8, 32 or 64, a whole one); rows whose g has two limbs and one; dx in one part and (cap 2048) in several;
# copies of w because of the type, the width and (offset 1) the address
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("cap,dtype,rows,width,vocab",
                         [(256, *c) for c in (("bf16", 1, 64, 600), ("bf16", 100, 72, 777), ("bf16", 300, 96, 1000), ("bf16", 300, 67, 1003), ("bf16", 40, 33, 513), ("bf16", 1100, 136, 1537),
                                              ("f32", 1, 40, 515), ("f32", 40, 33, 768), ("f32", 130, 72, 777), ("f32", 1100, 40, 801), ("bf16", 9000, 24, 600))] +
                         [(2048, *c) for c in (("bf16", 200, 64, 5003), ("bf16", 60, 515, 4500), ("f32", 150, 40, 5003), ("f32", 20, 70, 8200), ("bf16", 20, 67, 8200))])
def test_small_pieces(monkeypatch, cap, dtype, rows, width, vocab, offset):
    print(f"linear_xent pieces of {cap} {rows} {width} {vocab} {dtype} offset {offset}", flush=True)
    whole = ng.ngc_linear_xent_workspace_bytes(CODE[dtype], rows, width, vocab, True)
    monkeypatch.setenv("NGC_XENT_PIECE", str(cap))
    assert ng.ngc_linear_xent_workspace_bytes(CODE[dtype], rows, width, vocab, True) < whole     # a piece's g and copy of w
    _check(dtype, *_inputs(dtype, rows, width, vocab, 101 + rows), offset=offset)


@pytest.mark.parametrize("dtype,rows,width,vocab", [("f32", 1000, 2048, 50257), ("bf16", 1000, 4098, 70001)])
def test_two_pieces_of_a_large_vocabulary(dtype, rows, width, vocab):
    print(f"linear_xent two pieces {rows} {width} {vocab} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(3)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn(rows, width, generator=gen, device="cuda").to(t)
    w = (torch.randn(vocab, width, generator=gen, device="cuda") * (2 / width ** 0.5)).to(t)
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    labels[:4] = torch.tensor([0, vocab - 1, -100, vocab], device="cuda")
    dloss = torch.rand(rows, generator=gen, device="cuda")
    loss, lse, dx, dw = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    code = CODE[dtype]
    ws = torch.empty(max(ng.ngc_linear_xent_workspace_bytes(code, rows, width, vocab, b) for b in (0, 1)), dtype=torch.uint8, device="cuda")
    ng.ngc_linear_xent(code, rows, width, vocab, x, w, labels, loss, lse, ws, stream())
    ng.ngc_linear_xent_bwd(code, rows, width, vocab, x, w, labels, lse, dloss, dx, dw, ws, stream())
    x, w = x.double(), w.double()
    z = x @ w.T.contiguous()
    want = torch.logsumexp(z, 1)
    live = (labels >= 0) & (labels < vocab)
    at, n = labels.clamp(0, vocab - 1), torch.arange(rows, device="cuda")
    # logits of 2 in the mean: sums of `width` products, (width + 2) 2^-24 sum |x w| = 2^-12 sqrt(width) at the very most; the sums err like a random walk
    assert (lse.double() - want).abs().max() <= 1e-4
    assert (loss.double() - torch.where(live, want - z[n, at], 0.0)).abs().max() <= 2e-4
    g = torch.exp(z - lse.double()[:, None])
    g[n, at] -= 1
    g *= torch.where(live, dloss.double(), 0.0)[:, None]
    bound = (2.0 ** -7 if dtype == "bf16" else 1e-5) + 1e-4      # two roundings of half a step (fp32: the sums'), and the logits' error
    for got, ref in ((dx, g @ w), (dw, g.T.contiguous() @ x)):
        assert (got.double() - ref).norm() <= bound * ref.norm()
        part = (got.double() - ref).norm(dim=1)                  # row by row: no piece is off
        assert (part <= 4 * bound * ref.norm(dim=1) + 1e-3 * ref.norm() / ref.shape[0] ** 0.5).all()
    assert bool((dx[~live] == 0).all())
