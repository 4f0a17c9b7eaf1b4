"""Sizes next to the limits of caches, attention and logits: indices close to 2^31, grids close to what a launch holds."""
import pytest
import torch

from cache_util import HostCache, assert_within, attention_reference, offsets, random_q

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
MOST = 2 ** 31 - 2                                                     # entries of a pattern


@pytest.fixture
def entries():
    """The column array of a pattern of as many entries as one may have (8.6 GB); a test fills its end."""
    crd = torch.full((MOST,), -5, dtype=torch.int32, device="cuda")
    yield crd
    del crd
    torch.cuda.empty_cache()


def test_rules_whose_entries_end_where_int32_does(entries):
    """A row's history, way and biases lie at the end of their arrays: more of each than the threads of a workgroup, and than it
    holds in registers."""
    import paper_1804_10112_amd as spt
    V, n = 5003, 4900
    entries[-n:] = torch.arange(n, dtype=torch.int32, device="cuda").flip(0)
    pos = i32([MOST - n, MOST])
    pattern = spt.DeviceCSR(pos, entries, V)
    values = torch.full((MOST,), 1e9, device="cuda")
    values[-n:] = 4.0
    logits = torch.randn(1, V, device="cuda")
    rules = spt.LogitRules(first=i32([0, 1]), seen=pattern, tree=pattern, drafts=i32([V - 1]), presence=torch.ones(1, device="cuda"),
                           bias=spt.DeviceCSR(pos, entries, V, values, unique=True))
    out = torch.empty_like(logits)
    spt.spt_adjust_logits(logits, rules, out)
    want = logits.clone()
    want[0, :n] -= 1
    want[0, V - 1] -= 1                                                # node 0 is on the row's way: column 0 of the last entry
    want[0, :n] += 4
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_heads", [2, 40])                           # tiles of 16 rows, and of more
def test_trees_whose_entries_end_where_int32_does(entries, dtype, q_heads):
    import paper_1804_10112_amd as spt
    host = HostCache([70], 16, 2, 64, dtype, seed=1)
    rows = [[0], [1, 0], [0, 2]]
    flat = [c for r in rows for c in r]
    entries[-5:] = i32(flat)
    pos = i32([MOST - 5 + p for p in offsets([len(r) for r in rows])])
    q = random_q(3, q_heads, 64, dtype, 1)
    cache = host.device()
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(3, q_heads, device="cuda")
    spt.spt_cache_attention(cache, 0, i32([0, 3]), spt.DeviceCSR(pos, entries, 3), q.cuda(), 0.125, out, lse,
                            cache.workspace(spt.SPT_CACHE_ATTENTION, q_heads))
    torch.cuda.synchronize()
    ref, ref_lse, bound, lse_bound = attention_reference(host, 0, [3], rows, q, 0.125)
    assert_within(out, ref, bound, "out")
    assert_within(lse, ref_lse, lse_bound, "lse")


@pytest.mark.parametrize("pages", [MOST, MOST - 1023, MOST - 2 ** 21])
def test_pools_of_as_many_pages_as_one_may_have(pages):
    """The free pages are the last ones; the pages' slots overlap (a stride of 0), of which extending without sharing moves none."""
    import paper_1804_10112_amd as spt
    refs = torch.ones(pages, dtype=torch.int32, device="cuda")
    refs[-3:], refs[5] = 0, 0
    pool = torch.zeros(8, device="cuda").as_strided((1, pages, 1, 1, 8), (8, 0, 8, 8, 1))
    cache = spt.DeviceCache(pool, pool, torch.full((3, 3), -1, dtype=torch.int32, device="cuda"), i32([0, 0, 0]), refs)
    refused = i32([-1])
    spt.spt_cache_extend(cache, i32([3, 2, 1]), refused, cache.workspace(spt.SPT_CACHE_EXTEND))
    assert cache.table.tolist() == [[5, pages - 3, pages - 2], [-1, -1, -1], [-1, -1, -1]]
    assert cache.len.tolist() == [3, 0, 0] and int(refused.item()) == 2
    spt.spt_cache_extend(cache, i32([0, 1, 1]), refused, cache.workspace(spt.SPT_CACHE_EXTEND))
    assert cache.table.tolist() == [[5, pages - 3, pages - 2], [pages - 1, -1, -1], [-1, -1, -1]] and int(refused.item()) == 1
    assert refs[-3:].tolist() == [1, 1, 1] and int(refs[5]) == 1
    del refs, cache
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows", [2 ** 22, 2 ** 23 + 5, 2 ** 24])
def test_logits_of_as_many_rows_as_there_may_be(rows):
    """More rows than workgroups of one launch, alone and as sequences of three."""
    import paper_1804_10112_amd as spt
    V = 3
    logits = torch.randint(-8, 8, (rows, V), device="cuda").float()
    tokens = torch.randint(0, V, (rows,), dtype=torch.int32, device="cuda")
    out = torch.full_like(logits, 7.0)
    presence = torch.arange(rows, device="cuda").remainder(5).float()
    spt.spt_adjust_logits(logits, spt.LogitRules(presence=presence, drafts=tokens), out)
    want = logits.clone()
    want[torch.arange(rows, device="cuda"), tokens.long()] -= presence
    assert torch.equal(out, want)
    sequences = rows // 3
    first = torch.arange(0, 3 * sequences + 1, 3, dtype=torch.int32, device="cuda")
    out.fill_(7.0)
    spt.spt_adjust_logits(logits, spt.LogitRules(first=first, presence=presence[:sequences].contiguous(), drafts=tokens), out)
    way = torch.nn.functional.one_hot(tokens[:3 * sequences].long(), V).view(sequences, 3, V).cumsum(1).view(-1, V) > 0
    want = logits[:3 * sequences] - way * presence[:sequences].repeat_interleave(3)[:, None]
    assert torch.equal(out[:3 * sequences], want) and bool((out[3 * sequences:] == 7).all())
