"""Refusals and workspace sizes of the operators over tokens and a vocabulary (CPU: nothing passes the validation)."""
import numpy as np
import pytest

import paper_1801_08058_amd as ng

P = 0x1000
BF, F32 = ng.NGC_BF16, ng.NGC_F32


def _args(names, kw):
    return [kw[n] for n in names]


EMB = ("dtype", "tokens", "vocab", "width", "scale", "table", "ids", "y")
EMB_BWD = ("dtype", "tokens", "vocab", "width", "scale", "dy", "ids", "dtable", "ws")
NORM = ("dtype", "rows", "cols", "eps", "x", "gamma", "beta", "y", "mean", "rstd")
NORM_BWD = ("dtype", "rows", "cols", "x", "gamma", "mean", "rstd", "dy", "dx", "dgamma", "dbeta", "ws")
XENT = ("dtype", "rows", "width", "vocab", "x", "w", "labels", "loss", "lse", "ws")
XENT_BWD = ("dtype", "rows", "width", "vocab", "x", "w", "labels", "lse", "dloss", "dx", "dw", "ws")
CALLS = {"ngc_embedding": EMB, "ngc_embedding_bwd": EMB_BWD, "ngc_layer_norm": NORM, "ngc_layer_norm_bwd": NORM_BWD, "ngc_linear_xent": XENT,
         "ngc_linear_xent_bwd": XENT_BWD}
SIZES = {"tokens": 4, "rows": 4, "vocab": 10, "width": 8, "cols": 8, "scale": 1.0, "eps": 1e-5}


def _call(name, **kw):
    """The call with every argument valid except those given (and a workspace that is too small, so that nothing is launched)."""
    full = {n: SIZES.get(n, P) for n in CALLS[name]}
    full["dtype"], full["ws"] = BF, None
    full.update(kw)
    return getattr(ng, name)(*_args(CALLS[name], full), None, check=False)


@pytest.mark.parametrize("name", CALLS)
def test_types_and_sizes_are_refused(name):
    names = CALLS[name]
    for dtype in (-1, 2, 7):
        assert _call(name, dtype=dtype) == ng.NGC_BAD_ARG
    rows = "tokens" if "tokens" in names else "rows"
    cols = "width" if "width" in names else "cols"
    for bad in (0, -1, 1 << 31, 1 << 40):
        assert _call(name, **{rows: bad}) == ng.NGC_BAD_SHAPE
    for bad in (0, -5, 1 << 31, (1 << 32) + 8):                  # the last is 8 in 32 bits
        assert _call(name, **{cols: bad}) == ng.NGC_BAD_SHAPE
        if "vocab" in names:
            assert _call(name, vocab=bad) == ng.NGC_BAD_SHAPE
    assert _call(name, **{rows: 1 << 30, cols: 1 << 10}) == ng.NGC_BAD_SHAPE
    if "vocab" in names:
        assert _call(name, vocab=1 << 30, **{cols: 1 << 10}) == ng.NGC_BAD_SHAPE


@pytest.mark.parametrize("name", CALLS)
def test_pointers_are_refused(name):
    optional = {"gamma", "beta", "mean", "rstd", "dgamma", "dbeta", "dx", "dw"}
    if name == "ngc_layer_norm_bwd":
        optional -= {"mean", "rstd", "dx"}
    for n in CALLS[name]:
        if n in SIZES or n in ("dtype", "ws"):
            continue
        if n not in optional:
            assert _call(name, **{n: None}) == ng.NGC_BAD_ARG, n
        assert _call(name, **{n: P + 1}) == ng.NGC_BAD_ARG, n    # not element aligned
        if n in ("ids", "labels"):
            assert _call(name, **{n: P + 4}) == ng.NGC_BAD_ARG, n
        elif n not in ("table", "y", "x", "w", "dy", "dx", "dw"):
            assert _call(name, **{n: P + 2}) == ng.NGC_BAD_ARG, n
        elif n != "y" or name != "ngc_embedding":
            assert _call(name, dtype=F32, **{n: P + 2}) == ng.NGC_BAD_ARG, n
    if "ws" in CALLS[name]:
        assert _call(name, ws=P + 8) == ng.NGC_BAD_ARG


def test_workspaces_that_are_too_small_are_refused():
    for name in ("ngc_layer_norm_bwd", "ngc_linear_xent", "ngc_linear_xent_bwd"):
        assert _call(name) == ng.NGC_WORKSPACE_TOO_SMALL
        small = np.zeros(4, np.uint8)

        class Tensor:
            data_ptr = lambda self: P
            numel = lambda self: small.size
            element_size = lambda self: 1
        assert _call(name, ws=Tensor()) == ng.NGC_WORKSPACE_TOO_SMALL
    assert _call("ngc_linear_xent_bwd", dx=None, dw=None) == ng.NGC_BAD_ARG


def test_eps_and_vocabulary_limits():
    for eps in (-1e-5, float("nan"), float("inf"), float("-inf")):
        assert _call("ngc_layer_norm", eps=eps) == ng.NGC_BAD_ARG
    assert _call("ngc_embedding_bwd", vocab=(1 << 21) + 1) == ng.NGC_BAD_SHAPE
    assert ng.ngc_embedding_workspace_bytes(4, (1 << 21) + 1, 8) == 0


def test_workspace_queries():
    for bad in ((0, 10, 8), (4, 0, 8), (4, 10, 0), (1 << 31, 10, 8)):
        assert ng.ngc_embedding_workspace_bytes(*bad) == 0
    assert ng.ngc_layer_norm_workspace_bytes(9, 4, 8) == ng.ngc_layer_norm_workspace_bytes(BF, 0, 8) == 0
    assert ng.ngc_linear_xent_workspace_bytes(9, 4, 8, 10) == ng.ngc_linear_xent_workspace_bytes(BF, 4, 8, 0) == 0
    assert ng.ngc_layer_norm_workspace_bytes(BF, 4, 8) > 0
    for bwd in (False, True):
        assert ng.ngc_linear_xent_workspace_bytes(BF, 4, 8, 10, bwd) > 0
        # the logits of a large vocabulary do not fit what is asked for
        assert ng.ngc_linear_xent_workspace_bytes(BF, 65536, 512, 131072, bwd) < 65536 * 131072 * 2


def test_arguments_that_are_no_numbers_or_streams():
    for bad in ("s", object()):
        with pytest.raises(TypeError):
            ng.ngc_layer_norm(BF, 4, 8, bad, P, P, P, P, None, None, None, check=False)
        with pytest.raises(TypeError):
            ng.ngc_embedding(BF, 4, 10, 8, 1.0, P, P, P, bad, check=False)
