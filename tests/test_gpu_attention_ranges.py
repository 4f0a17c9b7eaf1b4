"""Attention at the ends of the numbers' range: weights far below the largest one, scores with a scale of 0."""
import math

import pytest
import torch

from cache_util import DTYPES, HALF_STEP, HostCache, gpu_attention

pytestmark = pytest.mark.gpu

SHAPES = [(1, 2), (20, 4), (70, 4)]                                     # drafts, query heads a head: tiles of 16, 64, 128 rows


def _rows_of_one_score(tokens, q_heads, width, dtype):
    q = torch.zeros(tokens, q_heads, width, dtype=DTYPES[dtype])
    q[:, :, 0] = 1
    return q


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("drafts,group", SHAPES)
@pytest.mark.parametrize("spread_out", [True, False])
@pytest.mark.parametrize("gap", [8.0, 14.0, 17.0, 18.0])
def test_many_tokens_far_below_one(dtype, drafts, group, spread_out, gap):
    """One token with a score of `gap`, 3000 of score 0: each of those weighs exp(-gap), up to 26 powers of two less. Its value is 0,
    so the result is the others' contribution alone. 40 sequences of 8 heads: a wave goes through hundreds of tokens after that one.

    A weight is rounded once to the values' type (half a step of it); in f16 one that is less than 2^-25 of the largest falls below
    the least normal number and is then off by at most 2^-36 of the largest. The exponential's argument is rounded to 32 bits where
    it is up to 38 (|gap| / ln 2 and 11), half a step of 2^-18, and its value to a step. Each sum of n positive numbers in 32 bits is off
    by (n - 1) 2^-24 of itself at most (exp(-17) added to 1 is less than half a step of it, and lost). The result is rounded once."""
    length, rows, heads, width = 3000, 40, 8, 8
    host = HostCache([length + drafts] * rows, 64, heads, width, dtype, poison=False, seed=drafts)
    host.K.zero_()
    host.V.abs_().add_(0.5)
    for s in range(rows):
        for h in range(heads):
            p, o = host.slot(s, (331 * s + 97 * h) % length if spread_out else 0)
            host.K[0, p, o, h, 0], host.V[0, p, o, h] = gap, 0
    out, lse = gpu_attention(host.device(), 0, [drafts] * rows, None, _rows_of_one_score(rows * drafts, group * heads, width, dtype), 1.0)
    pages = torch.tensor(host.table)[:, :host.held(length + drafts)]
    values = host.V[0][pages].reshape(rows, -1, heads, width)[:, :length + drafts].double()
    others = values.cumsum(1)[:, length:].flatten(0, 1).repeat_interleave(group, 1)     # of the tokens that each draft sees
    seen = torch.arange(length, length + drafts, dtype=torch.float64).repeat(rows)[:, None, None]
    small = math.exp(-gap)
    total = 1 + seen * small
    want = small * others / total
    h = HALF_STEP[dtype]
    exact = 2.0 ** -18 + 2.0 ** -22 + (length + drafts + 64) * 2.0 ** -24
    weights = exact + (0 if dtype == "f32" else h)
    lost = 2.0 ** -36 * others + 2.0 ** -25 if dtype == "f16" else 0
    error, bound = (out.double() - want).abs(), want * (2 * weights + h) + lost
    assert bool((error <= bound).all()), f"{float((error / bound).max())} times the bound"
    want_lse = gap + torch.log(total[:, :, 0])
    assert bool(((lse.double() - want_lse).abs() <= exact + 2.0 ** -23 * want_lse).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts,q_heads", SHAPES)
def test_a_scale_of_zero_weighs_scores_of_any_size_alike(dtype, drafts, q_heads):
    """z = 0 * score = 0 for every finite score, 3e37 too."""
    host = HostCache([200 + drafts], 16, 1, 64, dtype, poison=False, seed=3)
    host.K[..., 0] = torch.where(torch.rand(host.K.shape[:-1]) < 0.5, 1e19, -1e19).to(DTYPES[dtype])
    q = _rows_of_one_score(drafts, q_heads, 64, dtype) * 3e18
    out, lse = gpu_attention(host.device(), 0, [drafts], None, q, 0.0)
    pages = torch.tensor(host.table[0][:host.held(200 + drafts)])
    values = host.V[0][pages, :, 0].reshape(-1, 64)[:200 + drafts].double()
    seen = torch.arange(201, 201 + drafts, dtype=torch.float64)
    want = values.cumsum(0)[200:] / seen[:, None]
    spread = values.abs().cumsum(0)[200:] / seen[:, None]
    bound = (HALF_STEP[dtype] * want.abs() + (64 + 270) * 2.0 ** -23 * spread)[:, None]
    assert bool(((out.double() - want[:, None]).abs() <= bound).all())
    assert bool(((lse.double() - torch.log(seen)[:, None]).abs() <= (64 + 270) * 2.0 ** -23).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("drafts,q_heads", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_finite_scores_of_any_size(dtype, drafts, q_heads, sign):
    """One token's score is the largest by far more than any rounding, and as large as the type lets it be (keys of the type's lowest number
    among them): it has all the weight, so the result is its value and lse its score, off by its rounding in 32 bits.

    The score is a product of two numbers, exact or rounded once, times the scale; ln and log2 cost a few roundings more. Its weight w
    is rounded to the type once (half a step h; the sum of weights is w itself), the result w V / w once, and in 32 bits three times."""
    h = 0.0 if dtype == "f32" else HALF_STEP[dtype]
    largest = torch.finfo(DTYPES[dtype]).max
    for size in [1e3, 3e4, 6e4, largest] + ([] if dtype == "f16" else [1.1e7, 3e8, 7.7e9, 1e20, 1.2345e31, 3e37]):
        for factor in (0.37, 1.0, 60000.0 if dtype == "f16" else 1.9):
            # the other tokens' keys are a tenth of it: their scores less than half of the largest, or negative
            host = HostCache([300 + drafts], 16, 1, 64, dtype, poison=False, seed=3)
            q = _rows_of_one_score(drafts, q_heads, 64, dtype) * factor
            host.K.zero_()
            host.K[..., 0] = -sign * size
            host.K[0, :, ::2, 0, 0] = sign * size / 10
            best = 171                                                  # an odd slot of its page
            p, o = host.slot(0, best)
            host.K[0, p, o, 0, 0] = sign * size
            scale = sign * 0.9
            key, query = host.K[0, p, o, 0, 0].double(), q[0, 0, 0].double()
            score = float(key * query * torch.tensor(scale, dtype=torch.float32).double())
            if abs(score) * 1.4427 > 3e38:
                continue
            out, lse = gpu_attention(host.device(), 0, [drafts], None, q, scale)
            value = host.V[0, p, o].double()
            assert bool(((out.double() - value).abs() <= (2 * h + h * h + 2.0 ** -22) * value.abs()).all()), (size, factor)
            assert bool(((lse.double() - score).abs() <= 8 * 2.0 ** -24 * abs(score)).all()), (size, factor)


def test_all_scores_as_low_as_they_can_be():
    """Keys of the lowest number everywhere: all weigh alike, whatever their score."""
    for dtype in ("bf16", "f32"):
        for drafts, q_heads in SHAPES:
            host = HostCache([200 + drafts], 16, 1, 64, dtype, poison=False, seed=3)
            host.K.zero_()
            host.K[..., 0] = torch.finfo(DTYPES[dtype]).min
            q = _rows_of_one_score(drafts, q_heads, 64, dtype)
            out, lse = gpu_attention(host.device(), 0, [drafts], None, q, 0.3)
            pages = torch.tensor(host.table[0][:host.held(200 + drafts)])
            values = host.V[0][pages, :, 0].reshape(-1, 64)[:200 + drafts].double()
            seen = torch.arange(201, 201 + drafts, dtype=torch.float64)
            want = values.cumsum(0)[200:] / seen[:, None]
            spread = values.abs().cumsum(0)[200:] / seen[:, None]
            bound = (HALF_STEP[dtype] * want.abs() + (64 + 270) * 2.0 ** -23 * spread)[:, None]
            assert bool(((out.double() - want[:, None]).abs() <= bound).all()), dtype
            assert bool((lse < -1e37).all() and torch.isfinite(lse).all())
