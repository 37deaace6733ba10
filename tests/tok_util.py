"""Helpers of the tests of the operators over tokens: matrices with padded rows and bounds in 64 bits.

U[t] is half a step of type t relative to the value (one rounding), E32 the same of fp32.  TINY covers what is below the
smallest normal number of fp16.
"""
import zlib

import torch

from paper_2303_02191_b200 import binding as rt

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {k: torch.finfo(v).eps / 2 for k, v in DT.items()}
E32 = 2.0 ** -24
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}

_ctx = None


def ctx():
    global _ctx
    if _ctx is None:
        _ctx = rt.Context(0)
    return _ctx


class Rand:
    def __init__(self, *seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(zlib.crc32(repr(seed).encode()))

    def normal(self, rows, cols, std=1.0):
        return torch.empty(rows, cols, device="cuda").normal_(0.0, std, generator=self.g)


CANARY = 77.0


def matrix(src_or_shape, dtype, pad=0, to=16):
    """A matrix inside a wider and longer one full of canaries: rows start on 16-byte boundaries, `pad` more units of 16
    bytes lie between them.  -> (view, whole)"""
    rows, cols = src_or_shape if isinstance(src_or_shape, tuple) else src_or_shape.shape
    unit = max(1, to // torch.empty(0, dtype=dtype).element_size())
    width = (cols + unit - 1) // unit * unit + pad * unit
    whole = torch.full((rows + 2, width), CANARY, device="cuda").to(dtype)
    view = whole[:rows, :cols]
    if not isinstance(src_or_shape, tuple):
        view.copy_(src_or_shape)
    return view, whole


def untouched(view, whole):
    """What lies around the matrix is as it was."""
    rows, cols = view.shape
    return bool((whole[rows:] == CANARY).all()) and bool((whole[:rows, cols:] == CANARY).all())


def within(got, want, tol, what):
    """got inside want +- tol (64-bit tensors), no NaN."""
    d = (got.double() - want).abs()
    ok = d <= tol
    if not bool(ok.all()):
        worst = torch.argmax(torch.where(torch.isnan(d), torch.inf, d - tol))
        raise AssertionError("%s: %d of %d values off; worst got %r want %r tol %r" % (
            what, int((~ok).sum()), d.numel(), float(got.double().reshape(-1)[worst]), float(want.reshape(-1)[worst]), float(tol.reshape(-1)[worst])))
