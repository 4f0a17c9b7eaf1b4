"""Attention in each of its tiles: widths that do not fill one, values that are not finite, missing pages, many sequences."""
import math

import numpy as np
import pytest
import torch

from cache_util import DTYPES, HostCache, assert_within, attention_reference, check_attention, gpu_attention, random_q, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("width", [8, 40, 72, 120, 200])
@pytest.mark.parametrize("shaped", [True, False])
def test_widths_that_do_not_fill_a_tile_of_128_rows(dtype, width, shaped):
    """More than 256 rows a sequence (from 129 values on those are tiles of 64)."""
    counts = [140, 131]
    host = HostCache([c + n for c, n in zip(counts, (75, 0))], 16, 1, width, dtype, seed=width)
    check_attention(host, counts, random_tree(counts, width) if shaped else None, 2, seed=width, what=f"{dtype} {width}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("width", [8, 24, 56, 104, 136, 248])
def test_widths_that_do_not_fill_a_tile_of_64_rows(dtype, width):
    counts = [33, 20]
    host = HostCache([150, 40], 8, 2, width, dtype, seed=width)
    check_attention(host, counts, random_tree(counts, width), 4, seed=width, what=f"{dtype} {width}")


@pytest.mark.parametrize("width", [8, 24, 72, 136, 200, 248])
@pytest.mark.parametrize("drafts", [17, 40, 150])
def test_widths_that_do_not_fill_a_tile_of_32_rows_of_32_bits(width, drafts):
    counts = [drafts, drafts // 2 + 9]
    host = HostCache([drafts + 50, drafts + 9], 8, 1, width, "f32", seed=width)
    check_attention(host, counts, random_tree(counts, width), 1, seed=width, what=f"{width} {drafts}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("width", [64, 72, 128])
def test_values_that_are_not_finite_in_tiles_of_128_rows(dtype, bad, width):
    """In drafted tokens of the first, of a middle and of the last step: whoever does not see them is not reached by them."""
    context, drafts, places = 77, 300, (5, 130, 299)
    host = HostCache([context + drafts], 16, 1, width, dtype, seed=3)
    tree = random_tree([drafts], 5, roots=False)
    for j in places:
        p, o = host.slot(0, context + j)
        host.V[0, p, o, 0, [1, width - 1]] = bad
    q, scale = random_q(drafts, 1, width, dtype, 1), width ** -0.5
    out, lse = gpu_attention(host.device(), 0, [drafts], tree, q, scale)
    ref, ref_lse, bound, lse_bound = attention_reference(host, 0, [drafts], tree, q, scale)
    assert_within(lse, ref_lse, lse_bound, "lse")
    assert_within(out, ref, torch.nan_to_num(bound, nan=0.0, posinf=0.0), "out")
    clean = [i for i in range(drafts) if not set(places) & set(tree[i])]
    assert clean and len(clean) < drafts and bool(torch.isfinite(out[clean].float()).all())


@pytest.mark.parametrize("dtype,width", [("bf16", 128), ("f16", 64), ("bf16", 88)])
def test_missing_pages_in_tiles_of_128_rows(dtype, width):
    counts = [130, 135]
    host = HostCache([200, 191], 8, 1, width, dtype, seed=width)
    host.table[0][0], host.table[0][9], host.table[1][23], host.table[1][11] = -1, 1 << 20, -5, 10_000
    check_attention(host, counts, random_tree(counts, 3), 2, what="missing pages")
    check_attention(host, counts, None, 2, what="missing pages, no tree")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sequences", [63, 64, 65, 129, 300])
def test_many_sequences_of_many_rows(dtype, sequences):
    """A wave looks at 64 sequences at once for the beginning of its share; some have no drafted tokens, some no tokens at all."""
    rng = np.random.default_rng(sequences)
    counts = [0 if rng.random() < 0.3 else int(n) for n in rng.integers(1, 40, sequences)]
    lens = [n + (int(rng.integers(0, 60)) if n or rng.random() < 0.5 else 0) for n in counts]
    host = HostCache(lens, 16, 1, 32, dtype, seed=sequences)
    check_attention(host, counts, random_tree(counts, sequences), 3, what=f"{sequences}")


def test_many_sequences_of_hundreds_of_rows():
    counts = [60 if s % 3 else 0 for s in range(100)]
    host = HostCache([n + s % 50 for s, n in enumerate(counts)], 16, 1, 64, "bf16", seed=1)
    check_attention(host, counts, None, 8, what="tiles of 128 rows")
