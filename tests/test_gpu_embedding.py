"""ngc_embedding / ngc_embedding_bwd through the C ABI against the fp64 oracle.

Bounds, elementwise: a looked-up element is one fp32 product, rounded once to its type.  A gradient element is a sum of n fp32 terms in some
order, times scale: at most (n + 1) roundings of partial sums that are no larger than sum |dy| scale."""
import numpy as np
import pytest
import torch

import oracle
import paper_1801_08058_amd as ng
from tokens_util import CODE, HALF, TYPE, U, Guarded, stream, values, workspace, zipf_ids

pytestmark = pytest.mark.gpu


def _lookup(dtype, tokens, vocab, width, scale, ids, offset=0, seed=11):
    table = values(seed, 0, (vocab, width), 1.0, dtype)
    td, yd = Guarded(vocab * width, TYPE[dtype], offset, table), Guarded(tokens * width, TYPE[dtype], offset)
    idd = Guarded(tokens, torch.int64, 0, ids)
    ng.ngc_embedding(CODE[dtype], tokens, vocab, width, scale, td.t, idd.t, yd.t, stream())
    torch.cuda.synchronize()
    ref = oracle.embedding(table, ids, np.float32(scale))
    got = yd.f64(tokens, width)
    assert (np.abs(got - ref) <= np.abs(ref) * (HALF[dtype] + U) * 1.001).all()
    assert (got[(ids < 0) | (ids >= vocab)] == 0).all()
    assert yd.intact()


def _grad(dtype, tokens, vocab, width, scale, ids, offset=0, seed=12):
    dy = values(seed, 1, (tokens, width), 1.0, dtype)
    dyd, out = Guarded(tokens * width, TYPE[dtype], offset, dy), Guarded(vocab * width, torch.float32, offset)
    idd = Guarded(tokens, torch.int64, 0, ids)
    ws, behind = workspace(ng.ngc_embedding_workspace_bytes(tokens, vocab, width))
    ng.ngc_embedding_bwd(CODE[dtype], tokens, vocab, width, scale, dyd.t, idd.t, out.t, ws, stream())
    torch.cuda.synchronize()
    ref = oracle.embedding_bwd(dy, ids, vocab, np.float32(scale))
    mass = oracle.embedding_bwd(np.abs(dy), ids, vocab, abs(float(np.float32(scale))))
    count = np.bincount(ids[(ids >= 0) & (ids < vocab)], minlength=vocab)[:, None]
    got = out.f64(vocab, width)
    worst = np.abs(got - ref) - (count + 1) * U * 1.001 * mass
    assert (worst <= 0).all(), (worst.max(), np.unravel_index(worst.argmax(), worst.shape))
    assert out.intact() and bool((behind == 0xFF).all())
    # run to run
    again = Guarded(vocab * width, torch.float32, offset)
    ws.fill_(0)
    ng.ngc_embedding_bwd(CODE[dtype], tokens, vocab, width, scale, dyd.t, idd.t, again.t, ws, stream())
    torch.cuda.synchronize()
    assert torch.equal(again.t.view(torch.int32), out.t.view(torch.int32))


SIZES = [(1, 1, 1), (1, 300, 8), (2, 5, 7), (3, 1000, 64), (64, 17, 65), (65, 1000, 257), (300, 64, 1000), (129, 2048, 1024), (1000, 4099, 33),
         (700, 100, 2056), (33, 50257, 16), (5, 3, 8200), (260, 7, 520)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", SIZES)
def test_lookup(dtype, tokens, vocab, width):
    print(f"embedding {tokens} {vocab} {width} {dtype}", flush=True)
    ids = zipf_ids(tokens * 3 + vocab, tokens, vocab)
    _lookup(dtype, tokens, vocab, width, float(width) ** 0.5, ids)
    _lookup(dtype, tokens, vocab, width, -0.37, ids, offset=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", SIZES)
def test_gradient(dtype, tokens, vocab, width):
    print(f"embedding_bwd {tokens} {vocab} {width} {dtype}", flush=True)
    ids = zipf_ids(tokens * 5 + vocab, tokens, vocab)
    _grad(dtype, tokens, vocab, width, float(width) ** 0.5, ids)
    _grad(dtype, tokens, vocab, width, -0.37, ids, offset=1)


# many tokens: several blocks of the sort, rows with thousands of tokens, a vocabulary of more ranges than tokens
@pytest.mark.parametrize("dtype,tokens,vocab,width", [("bf16", 5001, 10007, 72), ("f32", 4097, 300, 40), ("bf16", 20000, 37, 24), ("bf16", 70000, 2000, 8),
                                                      ("f32", 2049, 131072, 5), ("bf16", 9000, 1 << 21, 2), ("bf16", 140001, 5000, 9)])
def test_gradient_of_many_tokens(dtype, tokens, vocab, width):
    print(f"embedding_bwd {tokens} {vocab} {width} {dtype}", flush=True)
    _grad(dtype, tokens, vocab, width, 1.5, zipf_ids(tokens + vocab, tokens, vocab))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["one", "none", "last", "descending", "two_hot"])
def test_gradient_where_ids_are_special(dtype, kind):
    tokens, vocab, width = 6000, 1000, 130
    ids = {"one": np.full(tokens, 7), "none": np.full(tokens, -100), "last": np.full(tokens, vocab - 1),
           "descending": (tokens - 1 - np.arange(tokens)) % vocab, "two_hot": np.where(np.arange(tokens) % 3 == 0, 5, 6)}[kind].astype(np.int64)
    print(f"embedding_bwd special {kind} {dtype}", flush=True)
    _grad(dtype, tokens, vocab, width, 1.0, ids)
    _lookup(dtype, tokens, vocab, width, 1.0, ids)


def test_ids_beyond_32_bits_are_outside_the_vocabulary():
    vocab, width = 50, 16
    ids = np.array([3, 3 + (1 << 32), -(1 << 40), 1 << 31, 4, np.iinfo(np.int64).min, np.iinfo(np.int64).max, 0], np.int64)
    _lookup("bf16", ids.size, vocab, width, 1.0, ids)
    _grad("bf16", ids.size, vocab, width, 1.0, ids)
