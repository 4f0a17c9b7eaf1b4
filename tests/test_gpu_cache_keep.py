"""Lists of tokens to keep that name more than a row has: what is out of range is skipped, the others are kept."""
import pytest
import torch

from cache_util import HostCache, offsets

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("many", [1, 70])
def test_tokens_to_keep_that_a_row_does_not_have_are_skipped(many):
    """Ordered lists with entries below 0 and beyond the drafted tokens, one or many of them."""
    import paper_1804_10112_amd as spt
    below, above = list(range(-many, 0)), list(range(50, 50 + many))
    counts = [4, 6, 5, 3, 0, 7, 50]
    lists = [below + [1] + above, below + [0, 2, 5], [1, 4] + above, below + above, above, [3], below + list(range(0, 50, 3)) + above]
    host = HostCache([n + c for n, c in zip(counts, [2, 9, 0, 5, 8, 1, 30])], 4, 2, 16, "f32", layers=2, seed=many)
    cache, first = host.device(), offsets(counts)
    keep = spt.DeviceCSR(i32(offsets([len(r) for r in lists])), i32([c for r in lists for c in r]), 50 + many, ordered=True, unique=True)
    spt.spt_cache_compact(cache, i32(first), keep)
    host.compact(first, [[c for c in r if 0 <= c < n] for r, n in zip(lists, counts)])
    host.assert_same(cache)
