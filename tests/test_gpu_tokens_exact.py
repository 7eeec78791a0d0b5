"""Sums over many rows of small whole numbers, which fp32 holds exactly in every order: not one row may be missing or counted twice.

Layer norm's dgamma and dbeta with mean 0 and rstd 1 are sum x dy and sum dy; the gradient of an embedding is the sum of dy per id.  All values are whole
numbers of at most two, the sums below 2^24."""
import pytest
import torch

import paper_1801_08058_amd as ng
from tokens_util import CODE, TYPE, stream

pytestmark = pytest.mark.gpu


def _whole(shape, most, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=gen, device="cuda", dtype=torch.int8).to(TYPE[dtype])


# past 2^31 elements; rows in registers of a wave and of a workgroup, on the vector grid and off it, beyond the registers, below a vector
@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 600_000, 4096), ("bf16", 300_001, 515), ("f32", 300_001, 515), ("bf16", 70_003, 2056), ("f32", 20_011, 4099), ("bf16", 9001, 16384),
                                             ("f32", 9001, 8193), ("bf16", 3001, 40_003), ("f32", 3001, 20_000), ("bf16", 1_000_003, 5), ("f32", 1_000_003, 3), ("f32", 100_003, 64)])
def test_layer_norm_sums_of_whole_numbers(dtype, rows, cols):
    print(f"layer_norm_bwd exact {rows} {cols} {dtype}", flush=True)
    x, dy = _whole((rows, cols), 1, dtype, rows), _whole((rows, cols), 1, dtype, cols)
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    step = 1 << 16
    want = [torch.zeros(cols, dtype=torch.float64, device="cuda") for _ in range(2)]
    for r in range(0, rows, step):                               # at most 65536 terms of one
        want[0] += (x[r:r + step].float() * dy[r:r + step].float()).sum(0).double()
        want[1] += dy[r:r + step].float().sum(0).double()
    dgamma, dbeta = torch.full((cols,), float("nan"), device="cuda"), torch.full((cols,), float("nan"), device="cuda")
    ws = torch.full((ng.ngc_layer_norm_workspace_bytes(CODE[dtype], rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")
    ng.ngc_layer_norm_bwd(CODE[dtype], rows, cols, x, None, mean, rstd, dy, dy, dgamma, dbeta, ws, stream())     # dx in the place of dy
    assert torch.equal(dgamma.double(), want[0]) and torch.equal(dbeta.double(), want[1])


# more than 2^20 tokens: a wave of the first sort goes through more than 256 of them
@pytest.mark.parametrize("dtype,tokens,vocab,width", [("bf16", 1_100_003, 5000, 24), ("f32", 1_100_003, 70_001, 3), ("bf16", (1 << 21) + 5, 300, 33), ("f32", 3_000_001, 1 << 21, 8),
                                                      ("bf16", 1_048_576, 1, 16)])
def test_embedding_sums_of_whole_numbers(dtype, tokens, vocab, width):
    print(f"embedding_bwd exact {tokens} {vocab} {width} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(tokens + vocab)
    ids = (torch.exp(torch.rand(tokens, generator=gen, device="cuda", dtype=torch.float64) * float(torch.log(torch.tensor(vocab + 1.0)))) - 1).long().clamp_(0, vocab - 1)
    dead = torch.rand(tokens, generator=gen, device="cuda") < 0.05
    ids[dead] = torch.where(torch.arange(tokens, device="cuda")[dead] % 2 == 0, -1, vocab)
    dy = _whole((tokens, width), 2, dtype, 5)
    live = (ids >= 0) & (ids < vocab)
    want = torch.zeros(vocab, width, dtype=torch.float64, device="cuda").index_add_(0, ids[live], dy[live].double()) * 0.5
    dtable = torch.full((vocab, width), float("nan"), device="cuda")
    ws = torch.full((ng.ngc_embedding_workspace_bytes(tokens, vocab, width),), 0xFF, dtype=torch.uint8, device="cuda")
    ng.ngc_embedding_bwd(CODE[dtype], tokens, vocab, width, 0.5, dy, ids, dtable, ws, stream())
    assert torch.equal(dtable.double(), want)
