"""A plain attention in 64 bits and how far a kernel's 32-bit one may be from it, for the tests of the operators over
dense caches."""
import math

import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def attend64(q, k, v, weight_step=2.0 ** -16):
    """q [G, D], k and v [n, D] (any float type): (output [G, D], weights [G, n], bound of the output, bound of a weight
    relative to itself) in 64 bits; n == 0: zeros.

    A logit is a sum of D products: in any order its rounding is at most D 2^-24 of the sum of their magnitudes, and two
    roundings of the scale; a weight 2^x moves by that much relative to itself, numerator and denominator, and by the
    exponential's own 2^-22 each, and the denominator by a sum of n terms, of which no chain is longer than n / 4 + 64: the
    four waves of a block have different keys, or (where they have different queries) each adds two at a time for a lane and its partner.  An
    output is a sum of n products of such weights, relative to the sum of the products' magnitudes.  weight_step: what
    the weights are off as a matrix product takes them: 2^-16 in two bf16 terms of 8 bits each, 2 2^-8 in one (half a
    step, 2^-8, of every weight in the numerator, and as much in the denominator, which adds up the rounded ones)."""
    n, D = k.shape
    q, k, v = q.double(), k.double(), v.double()
    if n == 0:
        z = torch.zeros_like(q)
        return z, torch.zeros((q.shape[0], 0), dtype=torch.float64, device=q.device), z, 0.0
    a = q @ k.t().contiguous() / math.sqrt(D)
    p = torch.softmax(a, dim=-1)
    size = float((q.abs() @ k.abs().t().contiguous()).max()) / math.sqrt(D)
    chain = (n / 4 + 64) * 2.0 ** -24
    rel = 2 * ((D + 2) * 2.0 ** -24 * size + 2.0 ** -22) + chain
    return p @ v, p, (p @ v.abs()) * (rel + chain + weight_step), rel


def worst(got, ref, bound, dtype):
    """The largest excess over the bound, with half a step of the storage type for the one rounding (2^-8 of a bf16
    value); at most 0 for a right result."""
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    return float(((got.double() - ref).abs() - (bound + step * (ref.abs() + bound) + 1e-30)).max())
