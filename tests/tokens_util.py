"""Helpers of the tests over tokens and a vocabulary: seeded values that an element type holds exactly, tensors inside a guarded
allocation (what lies in front of and behind them has to stay as it was), results as fp64."""
from __future__ import annotations

import numpy as np
import torch

import paper_1801_08058_amd as ng
import synth_inputs

CODE = {"bf16": ng.NGC_BF16, "f32": ng.NGC_F32}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}       # one rounding to the type, relative to the value
U = 2.0 ** -24                                       # one rounding of fp32 arithmetic
GUARD = 64                                           # elements


def values(seed, tid, shape, std, dtype, mean=0.0):
    v = synth_inputs.normal(seed, tid, shape, mean, std).astype(np.float32)
    return synth_inputs.bf16_bits_to_f32(synth_inputs.f32_to_bf16_bits(v)) if dtype == "bf16" else v


class Guarded:
    """A tensor of n elements at `offset` elements (of its own size) past a 16-byte boundary, between two guards."""

    def __init__(self, n, dtype, offset=0, fill=None):
        self.buf = torch.full((GUARD + offset + n + GUARD,), -77.0 if dtype.is_floating_point else -77, dtype=dtype, device="cuda")
        self.lo, self.hi = GUARD + offset, GUARD + offset + n
        self.t = self.buf[self.lo:self.hi]
        if fill is not None:
            self.t.copy_(torch.from_numpy(np.ascontiguousarray(fill).reshape(-1)).to(dtype))
        elif dtype.is_floating_point:
            self.t.fill_(float("nan"))

    def intact(self):
        return bool((self.buf[:self.lo] == -77).all()) and bool((self.buf[self.hi:] == -77).all())

    def f64(self, *shape):
        return self.t.double().cpu().numpy().reshape(shape)


def workspace(nbytes):
    """Exactly nbytes, filled with NaN patterns, with a guard behind it."""
    buf = torch.full((nbytes + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    return buf[:nbytes], buf[nbytes:]


def stream():
    return torch.cuda.current_stream().cuda_stream


def zipf_ids(seed, n, vocab, dead=0.1):
    """Token ids whose frequency falls with the rank; a part of them outside the vocabulary, on both sides."""
    rng = np.random.default_rng(seed)
    ids = np.clip(np.exp(rng.random(n) * np.log(vocab + 1)).astype(np.int64) - 1, 0, vocab - 1)
    out = rng.random(n)
    ids[out < dead / 2] = -1 - rng.integers(0, 200)
    ids[(out >= dead / 2) & (out < dead)] = vocab + rng.integers(0, 2)
    return ids
