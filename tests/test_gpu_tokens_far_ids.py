"""Ids and labels outside the vocabulary at the ends of 64 bits, and those that are inside it in their lower 32 bits: padding like -1."""
import pytest
import torch

import paper_1801_08058_amd as ng
from tokens_util import CODE, TYPE, stream

pytestmark = pytest.mark.gpu
FAR = [-(1 << 63), (1 << 63) - 1, 1 << 32, (1 << 32) + 3, -(1 << 32), -(1 << 32) + 3, 1 << 31, (1 << 31) - 1, -(1 << 31), (1 << 63) - (1 << 32) + 1, -(1 << 63) + 255]


def _ids(n, vocab, far):
    ids = torch.arange(n, device="cuda") * 7 % vocab
    dead = torch.arange(n, device="cuda") % 3 == 1
    values = torch.tensor(FAR if far else [-1], device="cuda")
    ids[dead] = values[torch.arange(int(dead.sum()), device="cuda") % len(values)]
    return ids


def _data(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(TYPE[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", [(100, 50, 24), (9001, 1 << 20, 3), (40_000, 3000, 40)])
def test_far_ids_have_no_row(dtype, tokens, vocab, width):
    print(f"embedding far ids {tokens} {vocab} {width} {dtype}", flush=True)
    table, dy = _data((vocab, width), dtype, 1), _data((tokens, width), dtype, 2)
    ws = torch.empty(max(16, ng.ngc_embedding_workspace_bytes(tokens, vocab, width)), dtype=torch.uint8, device="cuda")
    got = []
    for far in (False, True):
        ids = _ids(tokens, vocab, far)
        y, dtable = torch.full_like(dy, float("nan")), torch.full((vocab, width), float("nan"), device="cuda")
        ng.ngc_embedding(CODE[dtype], tokens, vocab, width, 2.0, table, ids, y, stream())
        ng.ngc_embedding_bwd(CODE[dtype], tokens, vocab, width, 2.0, dy, ids, dtable, ws, stream())
        got.append((y, dtable))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert bool((got[1][0][ids != torch.arange(tokens, device="cuda") * 7 % vocab] == 0).all()) and bool(torch.isfinite(got[1][1]).all())


# the logits in parts, in tiles, in pieces of the vocabulary, straight from memory
@pytest.mark.parametrize("dtype,rows,width,vocab,cap", [("bf16", 100, 512, 500, None), ("bf16", 1100, 40, 3001, None), ("bf16", 1100, 40, 3001, 256), ("f32", 200, 33, 1003, 256),
                                                        ("bf16", 20, 67, 9001, None), ("f32", 20, 64, 9001, None), ("bf16", 9001, 24, 300, None)])
def test_far_labels_do_not_count(monkeypatch, dtype, rows, width, vocab, cap):
    print(f"linear_xent far labels {rows} {width} {vocab} {dtype} {cap}", flush=True)
    if cap:
        monkeypatch.setenv("NGC_XENT_PIECE", str(cap))
    x, w = _data((rows, width), dtype, 3), _data((vocab, width), dtype, 4) / width ** 0.5
    w = w.to(TYPE[dtype])
    dloss = torch.rand(rows, device="cuda")
    ws = torch.empty(max(ng.ngc_linear_xent_workspace_bytes(CODE[dtype], rows, width, vocab, b) for b in (0, 1)), dtype=torch.uint8, device="cuda")
    got = []
    for far in (False, True):
        labels = _ids(rows, vocab, far)
        loss, lse, dx, dw = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda"), torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
        ng.ngc_linear_xent(CODE[dtype], rows, width, vocab, x, w, labels, loss, lse, ws, stream())
        ng.ngc_linear_xent_bwd(CODE[dtype], rows, width, vocab, x, w, labels, lse, dloss, dx, dw, ws, stream())
        got.append((loss, lse, dx, dw))
    for a, b in zip(*got):
        assert torch.equal(a, b) and bool(torch.isfinite(b).all())
    dead = (labels < 0) | (labels >= vocab)
    assert bool((loss[dead] == 0).all()) and bool((dx[dead] == 0).all())
