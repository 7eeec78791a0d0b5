"""Operators over tokens and a vocabulary on tensors past 2^31 elements or bytes: rows at both ends, against torch on those rows."""
import pytest
import torch

import paper_1801_08058_amd as ng
from tokens_util import stream

pytestmark = pytest.mark.gpu


def _randn(*shape, seed, dtype=torch.bfloat16, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen).mul_(std)


def test_embedding_of_a_table_past_2_31_elements():
    vocab, width, tokens = 1 << 20, 2056, 4000                   # 2.16e9 elements
    table = _randn(vocab, width, seed=1)
    ids = torch.randint(0, vocab, (tokens,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    ids[:4] = torch.tensor([0, vocab - 1, vocab, -1], device="cuda")
    y = torch.empty(tokens, width, dtype=torch.bfloat16, device="cuda")
    print("embedding 2^20 x 2056", flush=True)
    ng.ngc_embedding(ng.NGC_BF16, tokens, vocab, width, 0.5, table, ids, y, stream())
    live = (ids >= 0) & (ids < vocab)
    assert torch.equal(y, torch.where(live[:, None], table[ids.clamp(0, vocab - 1)] * 0.5, torch.zeros((), dtype=torch.bfloat16, device="cuda")))
    del table
    dy = _randn(tokens, width, seed=3)
    dtable = torch.full((vocab, width), float("nan"), device="cuda")
    ws = torch.empty(ng.ngc_embedding_workspace_bytes(tokens, vocab, width), dtype=torch.uint8, device="cuda")
    ids[10:300] = vocab - 1                                      # a frequent id in the last row
    ng.ngc_embedding_bwd(ng.NGC_BF16, tokens, vocab, width, 0.5, dy, ids, dtable, ws, stream())
    live = (ids >= 0) & (ids < vocab)
    for v in (0, int(ids[500]), vocab - 1):
        want = dy[(ids == v) & live].double().sum(0) * 0.5
        mass = dy[(ids == v) & live].double().abs().sum(0) * 0.5
        assert ((dtable[v].double() - want).abs() <= 300 * 2.0 ** -24 * mass).all(), v
    touched = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    touched[ids[live]] = True
    assert bool(torch.isfinite(dtable.amax(1)).all()) and bool((dtable.abs().amax(1)[~touched] == 0).all())


def test_layer_norm_of_rows_past_2_31_elements():
    rows, cols = 600_000, 4096                                   # 2.46e9 elements
    x, dy = _randn(rows, cols, seed=4), _randn(rows, cols, seed=5)
    gamma, beta = torch.rand(cols, device="cuda") + 0.5, torch.rand(cols, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    print("layer_norm 600000 x 4096", flush=True)
    ng.ngc_layer_norm(ng.NGC_BF16, rows, cols, 1e-5, x, gamma, beta, y, mean, rstd, stream())
    at = torch.tensor([0, 1, 299_999, 524_287, 524_288, rows - 2, rows - 1], device="cuda")
    a = x[at].double()
    m = a.mean(1, keepdim=True)
    rs = 1 / ((a - m).pow(2).mean(1, keepdim=True) + 1e-5).sqrt()
    want = (a - m) * rs * gamma.double() + beta.double()
    assert ((y[at].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16).all()
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(ng.ngc_layer_norm_workspace_bytes(ng.NGC_BF16, rows, cols), dtype=torch.uint8, device="cuda")
    ng.ngc_layer_norm_bwd(ng.NGC_BF16, rows, cols, x, gamma, mean, rstd, dy, dx, dgamma, dbeta, ws, stream())
    g, xh = dy[at].double() * gamma.double(), (a - m) * rs
    want = rs * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    assert ((dx[at].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16).all()
    sums = sum(dy[r:r + 50_000].double().sum(0) for r in range(0, rows, 50_000))
    # 600000 terms of about one in fp32: 512 workgroups' sums of about 1200 rows each
    assert (dbeta.double() - sums).abs().max() <= (1200 + 600) * 2.0 ** -24 * rows


@pytest.mark.parametrize("rows", [3, 300])
def test_linear_xent_of_a_weight_past_2_31_elements(rows):
    width, vocab = 2048, (1 << 20) + 4099                        # w: 2.16e9 elements, 4.3 GB
    x, w = _randn(rows, width, seed=6), _randn(vocab, width, seed=7, std=0.02)
    labels = torch.full((rows,), vocab - 1, device="cuda")
    labels[1] = 0
    labels[2] = -100
    loss, lse, dloss = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.ones(rows, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(max(ng.ngc_linear_xent_workspace_bytes(ng.NGC_BF16, rows, width, vocab, b) for b in (0, 1)), dtype=torch.uint8, device="cuda")
    print(f"linear_xent {rows} x 2048 x {vocab}", flush=True)
    ng.ngc_linear_xent(ng.NGC_BF16, rows, width, vocab, x, w, labels, loss, lse, ws, stream())
    ng.ngc_linear_xent_bwd(ng.NGC_BF16, rows, width, vocab, x, w, labels, lse, dloss, dx, dw, ws, stream())
    z = torch.cat([x.float() @ w[v:v + 65536].float().T for v in range(0, vocab, 65536)], 1).double()
    want = torch.logsumexp(z, 1)
    assert (lse.double() - want).abs().max() <= 1e-4             # logits of about one: sums of 2048 fp32 products, 2048 2^-24 sum|x w| = 1e-4 at most
    at = labels.clamp(0, vocab - 1)
    ok = labels >= 0
    assert (loss.double() - torch.where(ok, want - z[torch.arange(rows, device="cuda"), at], 0.0)).abs().max() <= 2e-4
    g = torch.exp(z - lse.double()[:, None])
    g[torch.arange(rows, device="cuda"), at] -= 1
    g[~ok] = 0
    ref = sum(g[:, v:v + 65536].float() @ w[v:v + 65536].float() for v in range(0, vocab, 65536)).double()
    assert (dx.double() - ref).norm() <= 2.0 ** -7 * ref.norm()
    assert bool((dx[2] == 0).all())
    for lo, hi in ((0, 64), (vocab - 64, vocab), (1 << 19, (1 << 19) + 64)):
        ref = g[:, lo:hi].T @ x.double()
        assert (dw[lo:hi].double() - ref).norm() <= 2.0 ** -7 * ref.norm()
