"""Attention over a paged cache against its definition in float64: types, head layouts, lengths, pages, trees, masked places."""
import math

import numpy as np
import pytest
import torch

from cache_util import (DTYPES, HostCache, attention_reference, assert_within, check_attention, gpu_attention, offsets, pattern,
                        random_q, random_tree)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("width", [8, 16, 24, 64, 80, 96, 128, 136, 192, 256])
def test_widths(dtype, width):
    host = HostCache([70, 33, 129], 16, 2, width, dtype, seed=width)
    check_attention(host, [1, 3, 2], None, 4, seed=width, what=f"{dtype} {width}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,q_heads", [(1, 1), (1, 7), (3, 3), (2, 16), (8, 8), (1, 40), (4, 12)])
def test_head_groups(dtype, heads, q_heads):
    host = HostCache([61, 200, 5], 8, heads, 64, dtype, seed=heads)
    check_attention(host, [2, 5, 5], random_tree([2, 5, 5], 1), q_heads, what=f"{heads} {q_heads}")


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 500, 1025])
def test_lengths_of_one_row(length):
    host = HostCache([length], 16, 1, 64, "bf16", seed=length)
    check_attention(host, [1], None, 4, what=str(length))


@pytest.mark.parametrize("page", [1, 2, 4, 32, 64, 256, 2048])
@pytest.mark.parametrize("layout", ["slots", "heads"])
def test_page_sizes(page, layout):
    host = HostCache([130, 1, 77, 300], page, 2, 64, "f16", seed=page)
    check_attention(host, [5, 1, 7, 40], random_tree([5, 1, 7, 40], page), 4, layout=layout, what=f"{page} {layout}")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("drafts", [1, 2, 4, 8, 9, 16, 17, 31, 33, 64, 65, 130])
def test_trees_of_drafted_tokens(dtype, drafts):
    lens, counts = [drafts + 90, drafts, drafts + 3], [drafts, drafts, drafts // 2]
    host = HostCache(lens, 16, 2, 64, dtype, seed=drafts)
    check_attention(host, counts, random_tree(counts, drafts), 8, what=f"tree {drafts}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts", [3, 40, 150, 300])
def test_a_chunk_without_a_tree_sees_what_lies_before(dtype, drafts):
    counts = [drafts, drafts // 3]
    host = HostCache([drafts + 37, drafts // 3], 16, 2, 128, dtype, seed=drafts)
    check_attention(host, counts, None, 4, what=f"chunk {drafts}")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_that_see_nothing(dtype):
    """No context and no entries in the pattern: zeros and -infinity. Rows without drafted tokens or without any token at all."""
    lens, counts = [4, 0, 50, 6, 1], [4, 0, 0, 6, 1]
    tree = [[], [0], [], [0, 1, 2, 3], [], [], [], [], [], [], []]
    host = HostCache(lens, 4, 2, 64, dtype)
    check_attention(host, counts, tree, 4, what="nothing seen")
    out, lse = gpu_attention(host.device(), 0, counts, tree, random_q(11, 4, 64, dtype, 0), 0.1)
    assert bool((out[0] == 0).all()) and bool((lse[0] == -math.inf).all()) and bool((out[4:] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("context,drafts", [(0, 6), (45, 6), (45, 20), (0, 40), (77, 40), (100, 70)])
def test_what_a_token_does_not_see_does_not_reach_it(dtype, bad, context, drafts):
    """Infinities and NaNs in keys and values of drafted tokens that some see and others do not; every draft sees itself, so the
    bad one's own row is bad, and those below it."""
    host = HostCache([context + drafts, 20], 8, 2, 64, dtype, seed=3)
    counts, tree = [drafts, 2], random_tree([drafts, 2], 5, roots=False)
    for which, j in (("K", 2), ("V", 4), ("V", drafts - 1)):
        p, o = host.slot(0, context + j)
        getattr(host, which)[0, p, o, :, 3] = bad
    q = random_q(sum(counts), 4, 64, dtype, 1).abs() + 0.25      # a score of an infinite key is an infinity of its sign
    q = q.to(DTYPES[dtype])
    scale = 0.125
    out, lse = gpu_attention(host.device(), 0, counts, tree, q, scale)
    ref, ref_lse, bound, lse_bound = attention_reference(host, 0, counts, tree, q, scale)
    clean = [i for i in range(sum(counts)) if i >= drafts or not {2, 4, drafts - 1} & set(tree[i])]
    assert clean and len(clean) < sum(counts)
    assert_within(out[clean], ref[clean], bound[clean], "clean rows")
    assert_within(lse[clean], ref_lse[clean], lse_bound[clean], "clean rows' lse")
    values_only = [i for i in range(drafts) if 2 not in tree[i]]
    got = out[values_only].double()
    want = ref[values_only]
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isfinite(want) & ~torch.isnan(want)],
                                                                           want[~torch.isfinite(want) & ~torch.isnan(want)])


def test_scores_of_minus_infinity_weigh_nothing():
    host = HostCache([40], 8, 1, 64, "f32", seed=2)
    for t in (0, 7, 31):
        p, o = host.slot(0, t)
        host.K[0, p, o, 0, 0] = -math.inf
    q = random_q(3, 1, 64, "f32", 2).abs() + 0.1
    check_attention(host, [3], None, 1, q=q, what="-inf scores")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores up to a few hundred: the running maximum has to carry them."""
    host = HostCache([300, 90], 16, 2, 64, dtype, seed=4)
    host.K.mul_(8)
    check_attention(host, [3, 9], None, 4, scale=1.0, what="large scores")


def test_pages_outside_the_pool_hold_no_tokens():
    for dtype in ("bf16", "f32"):
        host = HostCache([100, 64, 30], 16, 2, 64, dtype, seed=9)
        host.table[0][2], host.table[0][6], host.table[1][0], host.table[2] = -1, 10_000, -7, [99] * host.width
        check_attention(host, [3, 2, 2], random_tree([3, 2, 2], 2), 4, what="bad pages")


def test_lengths_outside_the_table():
    """A length below the drafted tokens: those of negative places are not there. Beyond the table: the table's end."""
    host = HostCache([10, 40, 20], 4, 1, 64, "f32", seed=1, room=0)
    host.len[0], counts = 3, [5, 2, 2]
    check_attention(host, counts, [[0, 1, 2], [2], [2, 3], [4], [0, 1], [0], [0, 1], [0], [0, 1]], 2, what="short")
    cache = host.device()
    q = random_q(9, 2, 64, "f32", 0)
    host.len[1] = cache.c.row_pages * 4
    ref = gpu_attention(host.device(), 0, counts, None, q, 0.1)
    cache.len[1] = 2 ** 30
    cache.len[2] = -5
    got = gpu_attention(cache, 0, counts, None, q, 0.1)
    assert torch.equal(ref[0][:7], got[0][:7]) and bool((got[0][7:] == 0).all())


def test_columns_of_a_pattern_in_any_order_repeated_or_outside():
    host = HostCache([30, 12], 8, 2, 64, "bf16", seed=5)
    counts = [4, 12]
    tree = [[0, 0, 0], [1, 0], [3, 1, 3, 2], [9, -1, 4, 2]] + [[11 - i, 500, 0, 0] for i in range(12)]
    check_attention(host, counts, tree, 4, what="unordered pattern")


@pytest.mark.parametrize("dtype,length,drafts,q_heads,heads", [("bf16", 70_001, 3, 8, 2), ("f16", 20_011, 40, 8, 1), ("f32", 9000, 1, 2, 2)])
def test_long_rows(dtype, length, drafts, q_heads, heads):
    host = HostCache([length, 100, length // 7], 64, heads, 64, dtype, seed=6)
    counts = [drafts, drafts, 1]
    check_attention(host, counts, random_tree(counts, 6), q_heads, what="long")


def test_many_rows():
    rng = np.random.default_rng(8)
    lens = rng.integers(0, 90, 700).tolist()
    counts = [min(t, int(c)) for t, c in zip(lens, rng.integers(0, 4, 700))]
    host = HostCache(lens, 16, 1, 64, "bf16", seed=8)
    check_attention(host, counts, random_tree(counts, 8), 2, what="700 rows")


def test_strides_of_queries_and_results():
    """q and out as parts of wider tensors, heads before tokens; lse left out."""
    import paper_1804_10112_amd as spt
    host = HostCache([50, 21], 8, 2, 64, "bf16", seed=7)
    counts, q = [3, 2], random_q(5, 4, 64, "bf16", 7)
    ref, _, bound, _ = attention_reference(host, 0, counts, None, q, 0.2)
    cache = host.device()
    wide = torch.zeros(4, 5, 200, dtype=torch.bfloat16, device="cuda")
    qd = wide[:, :, 8:72].transpose(0, 1)
    qd.copy_(q)
    out = torch.full((5, 4, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    first = torch.tensor(offsets(counts), dtype=torch.int32, device="cuda")
    spt.spt_cache_attention(cache, 0, first, None, qd, 0.2, out[:, :, :64], None, cache.workspace(spt.SPT_CACHE_ATTENTION, 4))
    torch.cuda.synchronize()
    assert_within(out[:, :, :64], ref, bound, "strided")
    assert bool((out[:, :, 64:] == 7).all())


def test_offsets_beyond_32_bits():
    """A pool of which the used pages lie gigabytes apart."""
    import paper_1804_10112_amd as spt
    small = HostCache([60, 37], 16, 1, 64, "bf16", layers=2, spare=0, seed=3)
    pages, layers = small.K.shape[1], 2
    page_stride = 2 ** 28                                    # 512 MB in bf16
    layer_stride = page_stride * pages
    pool = torch.empty(layer_stride * layers, dtype=torch.bfloat16, device="cuda")
    cache = small.device()
    shape = small.K.shape
    views = [torch.as_strided(pool, shape, (layer_stride, page_stride, 64, 64, 1), off) for off in (0, 2 ** 20)]
    for view, data in zip(views, (small.K, small.V)):
        view.copy_(data.cuda())
    far = spt.DeviceCache(views[0], views[1], cache.table, cache.len, cache.refs)
    for layer, q_heads in ((0, 2), (1, 2), (1, 16), (0, 40)):       # one kernel for few rows, one for many
        q = random_q(5, q_heads, 64, "bf16", 3)
        near = gpu_attention(cache, layer, [3, 2], None, q, 0.1)
        got = gpu_attention(far, layer, [3, 2], None, q, 0.1)
        assert torch.equal(near[0], got[0]) and torch.equal(near[1], got[1])


def test_captured_and_replayed_while_the_row_grows():
    """One graph serves a row that grows and a tree that changes: lengths, first, pages and pattern are read on the device."""
    import paper_1804_10112_amd as spt
    host = HostCache([20, 130], 16, 2, 64, "bf16", spare=40, room=20, seed=11)
    counts = [3, 4]
    cache = host.device()
    q = random_q(7, 8, 64, "bf16", 11)
    tree_rows = random_tree(counts, 1)
    longest = offsets([i % 4 + 1 for i in range(7)])[-1]
    pos = torch.tensor(offsets([len(r) for r in tree_rows]), dtype=torch.int32, device="cuda")
    crd = torch.zeros(64, dtype=torch.int32, device="cuda")
    crd[:pos[-1].item()] = torch.tensor([c for r in tree_rows for c in r], dtype=torch.int32)
    tree = spt.DeviceCSR(pos, crd, 8)
    assert longest < 64
    first = torch.tensor(offsets(counts), dtype=torch.int32, device="cuda")
    qd, out = q.cuda(), torch.empty(7, 8, 64, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(7, 8, device="cuda")
    ws = cache.workspace(spt.SPT_CACHE_ATTENTION, 8)
    call = lambda: spt.spt_cache_attention(cache, 0, first, tree, qd, 0.125, out, lse, ws)
    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for step in range(4):
        if step:
            add = [17 * step, 5]
            assert host.extend(add) == 0
            for s, n in enumerate(add):                       # something in the new slots
                for t in range(host.len[s] - n, host.len[s]):
                    p, o = host.slot(s, t)
                    host.K[0, p, o], host.V[0, p, o] = torch.randn(2, 64).bfloat16(), torch.randn(2, 64).bfloat16()
            fresh = host.device()
            cache.K.copy_(fresh.K), cache.V.copy_(fresh.V), cache.table.copy_(fresh.table), cache.len.copy_(fresh.len)
            tree_rows = random_tree(counts, step)
            flat = [c for r in tree_rows for c in r]
            pos.copy_(torch.tensor(offsets([len(r) for r in tree_rows]), dtype=torch.int32))
            crd[:len(flat)] = torch.tensor(flat, dtype=torch.int32)
        out.fill_(math.nan), lse.fill_(math.nan), ws.fill_(255)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        ref, ref_lse, bound, lse_bound = attention_reference(host, 0, counts, tree_rows, q, 0.125)
        assert_within(out, ref, bound, f"replay {step}")
        assert_within(lse, ref_lse, lse_bound, f"replay {step} lse")
        replayed = out.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, replayed), "the eager call gives the same bits"


def test_two_streams_with_a_workspace_each():
    import paper_1804_10112_amd as spt
    host = HostCache([3000, 130], 16, 2, 128, "bf16", seed=12)
    cache, counts = host.device(), [5, 4]
    q = random_q(9, 8, 128, "bf16", 12)
    want = gpu_attention(cache, 0, counts, None, q, 0.1)
    first = torch.tensor(offsets(counts), dtype=torch.int32, device="cuda")
    qd = q.cuda()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(qd) for _ in range(2)]
    spaces = [cache.workspace(spt.SPT_CACHE_ATTENTION, 8) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for st, o, w in zip(streams, outs, spaces):
            spt.spt_cache_attention(cache, 0, first, None, qd, 0.1, o, None, w, stream=st)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o.cpu(), want[0])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0, 1e-30])
def test_scales(dtype, scale):
    """Negative ones turn the order round, 0 weighs everything seen alike."""
    for drafts in (2, 20, 60):
        counts = [drafts, 3]
        host = HostCache([drafts + 70, 9], 16, 2, 64, dtype, seed=drafts)
        check_attention(host, counts, random_tree(counts, 4), 4, scale=scale, what=f"scale {scale}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("drafts", [1, 17, 30, 70])
@pytest.mark.parametrize("width", [72, 128, 200])
def test_pages_that_are_missing_and_ends_of_steps(dtype, drafts, width):
    """Pages outside the pool at the beginning, within and at the end of a row, lengths around a step of 64 and 128 tokens."""
    for length in (drafts + 63, drafts + 64, drafts + 129):
        host = HostCache([length, length + 1], 8, 1, width, dtype, seed=length)
        host.table[0][0], host.table[0][5], host.table[1][(length + 1 - 1) // 8] = -1, 1 << 20, -5
        check_attention(host, [drafts, drafts], None, 2, what=f"{length} {drafts}")


def test_rows_of_very_different_sizes_in_one_call():
    """A chunk of a prompt beside rows that decode: one kernel serves both, whichever the mean chooses."""
    counts = [200] + [1] * 12 + [0] * 60 + [31]
    lens = [260] + [int(x) for x in np.random.default_rng(1).integers(1, 400, 12)] + [5] * 60 + [400]
    host = HostCache(lens, 16, 2, 64, "bf16", seed=1)
    check_attention(host, counts, None, 8, what="mixed, few")
    host = HostCache(lens[:3], 16, 2, 64, "bf16", seed=2)
    check_attention(host, counts[:3], None, 8, what="mixed, many")


def test_one_workspace_for_calls_of_several_shapes():
    """A workspace is scratch: calls of other sizes, with the same one, in turn give what each gives alone."""
    import paper_1804_10112_amd as spt
    host = HostCache([900, 40, 333], 16, 2, 128, "bf16", seed=5)
    cache = host.device()
    ws = cache.workspace(spt.SPT_CACHE_ATTENTION, 8)
    cases = []
    for counts in ([1, 1, 1], [40, 3, 9], [130, 40, 2], [5, 0, 0]):
        q = random_q(sum(counts), 8, 128, "bf16", sum(counts)).cuda()
        first = torch.tensor(offsets(counts), dtype=torch.int32, device="cuda")
        alone = torch.empty_like(q)
        spt.spt_cache_attention(cache, 0, first, None, q, 0.1, alone, None, cache.workspace(spt.SPT_CACHE_ATTENTION, 8))
        cases.append((q, first, alone))
    torch.cuda.synchronize()
    outs = [torch.empty_like(q) for q, _, _ in cases]
    for _ in range(3):
        for (q, first, _), out in zip(cases, outs):
            spt.spt_cache_attention(cache, 0, first, None, q, 0.1, out, None, ws)
    torch.cuda.synchronize()
    for (_, _, alone), out in zip(cases, outs):
        assert torch.equal(alone, out)


@pytest.mark.parametrize("counts", [[1, 1, 1], [40, 3, 9], [90, 40, 2]])
def test_results_in_place_of_the_queries(counts):
    import paper_1804_10112_amd as spt
    host = HostCache([700, 40, 333], 16, 2, 64, "bf16", seed=5)
    cache, q = host.device(), random_q(sum(counts), 8, 64, "bf16", 2)
    want = gpu_attention(cache, 0, counts, None, q, 0.1, extra=0)[0]
    first, qd = torch.tensor(offsets(counts), dtype=torch.int32, device="cuda"), q.cuda()
    spt.spt_cache_attention(cache, 0, first, None, qd, 0.1, qd, None, cache.workspace(spt.SPT_CACHE_ATTENTION, 8))
    torch.cuda.synchronize()
    assert torch.equal(qd.cpu(), want)
