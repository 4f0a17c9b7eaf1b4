"""Penalties at the ends of the types' ranges: quotients that overflow or underflow, repetitions below 1, infinities."""
import math

import pytest
import torch

from cache_util import DTYPES, HALF_STEP

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
REPETITIONS = [0.5, 0.85, 0.999, 1.0, 1.3, 3.0, 1e-3, 1e-30, 1e-38, 3e-39, 1e-39, 1e-45, 0.0, 1e20, 3e38, math.inf]


def _logits(dtype):
    """Powers of ten over the type's range, its largest and least numbers, infinities, zeros; with both signs."""
    info = torch.finfo(DTYPES[dtype])
    sizes = [10.0 ** e for e in range(-45, 39)] + [1.2345, 7.0, info.max, 0.97 * info.max, info.tiny, info.tiny * info.eps, math.inf, 0.0]
    x = torch.tensor(sizes, dtype=torch.float64).to(DTYPES[dtype])
    return torch.cat([x, -x])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_repetitions_at_both_ends_of_the_range(dtype):
    """x / repetition where x > 0, else x * repetition, in 32 bits, rounded to the type.

    The quotient is a product with one correction (or a division), off by at most two half steps of 32 bits; a result below the least
    normal number by one step there, 2^-149 in 32 bits and 2^-24 in f16, 2^-133 in bf16; what the largest number of a type cannot
    hold is an infinity. No result here lies within those errors of the largest number."""
    import paper_1804_10112_amd as spt
    x = _logits(dtype)
    V, N = x.numel(), len(REPETITIONS)
    logits = x.repeat(N, 1).cuda()
    repetition = torch.tensor(REPETITIONS, dtype=torch.float32)
    seen = spt.DeviceCSR(i32([V * s for s in range(N + 1)]), i32(list(range(V)) * N), V)
    out = torch.empty_like(logits)
    spt.spt_adjust_logits(logits, spt.LogitRules(seen=seen, repetition=repetition.cuda()), out)
    r, y = repetition.double()[:, None], x.double()[None, :]
    want = torch.where(y > 0, y / r, y * r)
    info, single = torch.finfo(DTYPES[dtype]), torch.finfo(torch.float32)
    infinite = want.abs() > info.max * (1 + HALF_STEP[dtype] / 2)
    want = torch.where(infinite, torch.sign(want) * math.inf, want)
    got = out.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
    fine = torch.isfinite(want)
    half = 0.0 if dtype == "f32" else HALF_STEP[dtype]
    least = single.tiny * single.eps + (0.0 if dtype == "f32" else info.tiny * info.eps)
    bound = want[fine].abs() * (half + 2 * 2.0 ** -24 * (1 + half)) + least
    assert bool(((got[fine] - want[fine]).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_quotient_beyond_the_largest_number_is_an_infinity(dtype):
    import paper_1804_10112_amd as spt
    largest = torch.finfo(DTYPES[dtype]).max
    logits = torch.tensor([[largest, -largest, 1.0]], dtype=DTYPES[dtype], device="cuda")
    rules = spt.LogitRules(seen=spt.DeviceCSR(i32([0, 3]), i32([0, 1, 2]), 3), repetition=torch.full((1,), 0.5, device="cuda"))
    spt.spt_adjust_logits(logits, rules, logits)
    assert logits.tolist() == [[math.inf, -largest / 2, 2.0]]
