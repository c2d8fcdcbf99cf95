"""Checks of the operators on 8-bit rows that tests share; tests/test_scaled_checks.py shows on the CPU what each of them catches."""
import torch

import scaled_ref as ref

F32, BF16 = torch.float32, torch.bfloat16


def residual_sum(h, y):
    """h + y in 64 bits, rounded once to h's type (past its largest: infinity)"""
    s = h.double() if y is None else ref.to_type(h.double() + y.double(), h.dtype)
    return torch.where(s.abs() >= 2.0 ** 128, torch.copysign(torch.full_like(s, float("inf")), s), s)


def same_values(got, want):
    """equal, and NaN in the same places"""
    got, want = got.double(), want.double()
    nan = want.isnan()
    return bool(torch.equal(got.isnan(), nan) and torch.equal(got[~nan], want[~nan]))


def beyond_rounding(got, want, dtype):
    """2-norm of what `got` is off by beyond half a step of its type, relative to that of `want` (64-bit)"""
    got = got.double()
    if not bool(torch.isfinite(got).all()):
        return float("inf")
    _, e = torch.frexp(want)                                             # want = f 2^e, f in [0.5, 1): a step is 2^(e - 24) or 2^(e - 8)
    half = 2.0 ** (e.double().clamp(min=-125) - (25 if dtype == F32 else 9))
    rest = ((got - want).abs() - half).clamp(min=0)
    return float(rest.norm() / want.norm().clamp(min=1e-300))


def sum_tolerance(k, dtype):
    """What the sums may be off by, 2-norm relative to the results', for inputs of random signs.

    Outputs in fp32: a sum of `blocks` blocks and of up to 16 parts, with four instructions a block, is rounded blocks + 21
    times, each by 2^-23 of it at most (rounded or cut), independently.
    Outputs in bf16: the instruction cuts seven products of an eight at 2^-13 of the largest at most: independent errors
    of up to 2^-13 max, uniform, are sqrt(7 / 3) 2^-13 of the largest together, which is at most what the eight's products
    are together (root of the sum of squares), and so of the whole."""
    blocks = ref.padded(k)[0]
    return (blocks + 21) ** 0.5 * 2.0 ** -23 + (0.0 if dtype == F32 else (7 / 3) ** 0.5 * 2.0 ** -13)


def one_binade(m, k, seed, powers=None):
    """[m][k] of +-1, 1.125 .. 1.875: what is held in 8 bits without loss, products of which in any eight lose nothing to a cut
    13 bits below the largest, and whose sums of up to 2^15 are exact in fp32 (22 bits)"""
    g = torch.Generator().manual_seed(seed)
    v = (8 + torch.randint(0, 8, (m, k), generator=g)).float() / 8
    v = torch.where(torch.rand(m, k, generator=g) < 0.5, -v, v)
    return v if powers is None else v * 2.0 ** powers.float()
