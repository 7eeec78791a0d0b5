"""What the switches for tests of the linear cross entropy do to its plan, seen in the workspace that it asks for (CPU)."""
import pytest

import paper_1801_08058_amd as ng
from tokens_util import CODE


def _without_logits(dtype, rows, width, vocab):
    """Bytes of the loss alone whose logits stay in tiles: a maximum and a sum per row and tile, the labels' logits, copies of the operands."""
    limbs, pitch = (3, -(-width // 32) * 32) if dtype == "f32" else (1, -(-width // 8) * 8)
    krows = -(-rows // 32) * 32 if dtype == "f32" else rows
    return rows * 8 * (-(-vocab // 64) + 1) + rows * 4 + krows * pitch * 2 * limbs + (-(-vocab // 32) * 32) * pitch * 2 * limbs + 4 * 256


# few tiles with long rows: by themselves they would run in parts, whose logits go through the workspace
@pytest.mark.parametrize("dtype,rows,width,vocab", [("bf16", 1, 8, 2), ("bf16", 257, 515, 1003), ("bf16", 300, 96, 777), ("bf16", 640, 264, 5003), ("bf16", 128, 2048, 1000), ("f32", 257, 515, 1003), ("f32", 130, 72, 300)])
def test_a_forced_tile_is_not_replaced_by_parts_of_another(monkeypatch, dtype, rows, width, vocab):
    monkeypatch.setenv("NGC_XENT_TILE", "256")
    assert ng.ngc_linear_xent_workspace_bytes(CODE[dtype], rows, width, vocab, False) <= _without_logits(dtype, rows, width, vocab)


def test_the_parts_of_few_tiles_are_there_without_the_switch():
    assert ng.ngc_linear_xent_workspace_bytes(ng.NGC_BF16, 128, 2048, 1000, False) >= _without_logits("bf16", 128, 2048, 1000) - 4 * 256 + 128 * 1000 * 4


def test_small_pieces_take_less(monkeypatch):
    whole = ng.ngc_linear_xent_workspace_bytes(ng.NGC_F32, 1100, 40, 8000, True)
    monkeypatch.setenv("NGC_XENT_PIECE", "256")
    assert ng.ngc_linear_xent_workspace_bytes(ng.NGC_F32, 1100, 40, 8000, True) < whole / 8
