"""Helpers of the tests of the operators on feature rows: tensors in awkward places, and how far an output may be off.

An output may be off by half a step of its type (once rounded) and by the rounding of 32-bit sums: `terms` roundings of at
most 2^-24 relative to the sum of the terms' magnitudes, which the oracle gives.
"""
import numpy as np
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNTOUCHED = 7.0


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def wide(t):
    return t.detach().cpu().double().numpy()


def near(got, ref, mag, terms, name=""):
    """got (a tensor) is ref to within its rounding; NaN in ref marks elements that the call leaves alone."""
    g = wide(got).reshape(ref.shape)
    alone = np.isnan(ref)
    assert np.all(g[alone] == UNTOUCHED), f"{name}: rows of no sequence were written"
    tol = half_step(got.dtype) * np.abs(ref) * (1 + 2.0 ** -7) + terms * 2.0 ** -24 * mag
    if got.dtype == torch.float16:
        tol = tol + 2.0 ** -25               # half a step of the subnormal numbers
    # A value beyond the type's largest number rounds to infinity, and a term beyond the largest 32-bit number does not exist in 32
    # bits; nor does a term whose factor is beyond it: a state of 2^-20 at least times an exponential.
    beyond = mag > min(torch.finfo(got.dtype).max, np.finfo(np.float32).max * 2.0 ** -20)
    bad = ~alone & ~beyond & ~(np.abs(g - ref) <= tol)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{name}: {bad.sum()} of {bad.size} off, first at {i}: {g[i]!r} for {ref[i]!r}, may be {tol[i]:.3g} off")


def matrix(values, dtype, pad=0, shift=0):
    """values [rows][width] on the GPU, in a matrix of `pad` more columns, the first `shift` of them in front."""
    values = torch.as_tensor(values)
    rows, width = values.shape
    m = torch.full((rows, width + pad), float("nan"), dtype=dtype, device="cuda")
    m[:, shift:shift + width] = values.to(dtype)
    return m[:, shift:shift + width]


def out_matrix(rows, width, dtype, pad=0, shift=0):
    return torch.full((rows, width + pad), UNTOUCHED, dtype=dtype, device="cuda")[:, shift:shift + width]


def surroundings_untouched(m):
    """The columns around a slice made by out_matrix still hold what they held."""
    base = m._base if m._base is not None else m
    keep = torch.ones_like(base, dtype=torch.bool)
    torch.as_strided(keep, m.size(), m.stride(), m.storage_offset()).fill_(False)
    return bool((base[keep].float() == UNTOUCHED).all())
