"""ngc_linear_xent_bwd of bf16 tensors with one limb of g at sizes that have two by themselves, and with two at one that has one (NGC_XENT_LIMBS): every
form of the products of both, against the fp64 oracle with the bounds of test_gpu_linear_xent.py."""
import pytest

import paper_1801_08058_amd as ng
from test_gpu_linear_xent import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("edge", [None, 64, 128, 256])
@pytest.mark.parametrize("rows,width,vocab", [(1, 8, 2), (3, 33, 63), (65, 72, 257), (130, 32, 1003), (128, 256, 1000), (33, 515, 777), (300, 40, 4099), (257, 515, 1003), (640, 264, 5003),
                                              (40, 1500, 4097), (16, 1030, 8193), (1100, 160, 3001), (9000, 24, 300)])
def test_one_limb(monkeypatch, rows, width, vocab, edge):
    print(f"linear_xent one limb {rows} {width} {vocab} edge {edge}", flush=True)
    two = ng.ngc_linear_xent_workspace_bytes(ng.NGC_BF16, rows, width, vocab, True)
    monkeypatch.setenv("NGC_XENT_LIMBS", "1")
    if edge:
        monkeypatch.setenv("NGC_XENT_TILE", str(edge))
    elif vocab < 8192:
        assert ng.ngc_linear_xent_workspace_bytes(ng.NGC_BF16, rows, width, vocab, True) <= two
    for offset in (0, 1):
        _check("bf16", *_inputs("bf16", rows, width, vocab, 111 + rows), offset=offset)


@pytest.mark.parametrize("cap", [256, 2048])
@pytest.mark.parametrize("rows,width,vocab", [(1, 64, 600), (200, 64, 5003), (300, 67, 2600), (1100, 136, 4097)])
def test_one_limb_in_pieces(monkeypatch, rows, width, vocab, cap):
    print(f"linear_xent one limb pieces of {cap} {rows} {width} {vocab}", flush=True)
    monkeypatch.setenv("NGC_XENT_LIMBS", "1")
    monkeypatch.setenv("NGC_XENT_PIECE", str(cap))
    _check("bf16", *_inputs("bf16", rows, width, vocab, 121 + rows))


def test_two_limbs_of_a_large_product(monkeypatch):
    rows, width, vocab = 600, 640, 9000
    one = ng.ngc_linear_xent_workspace_bytes(ng.NGC_BF16, rows, width, vocab, True)
    monkeypatch.setenv("NGC_XENT_LIMBS", "2")
    assert ng.ngc_linear_xent_workspace_bytes(ng.NGC_BF16, rows, width, vocab, True) > one
    _check("bf16", *_inputs("bf16", rows, width, vocab, 131))
