"""The pages of a cache against a host model of the same rules: extending, writing, compacting, freeing, forking."""
import numpy as np
import pytest
import torch

from cache_util import DTYPES, HostCache, offsets, pattern

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")


def _extend(host, cache, add, what=""):
    import paper_1804_10112_amd as spt
    refused = i32([-1])
    ws = cache.workspace(spt.SPT_CACHE_EXTEND)
    ws.fill_(255)
    spt.spt_cache_extend(cache, i32(add), refused, ws)
    want = host.extend(add)
    host.assert_same(cache, what)
    assert int(refused.item()) == want, what


@pytest.mark.parametrize("dtype,width", [("bf16", 64), ("f16", 8), ("f32", 80)])
@pytest.mark.parametrize("page", [1, 4, 16, 128])
@pytest.mark.parametrize("layout", ["slots", "heads"])
def test_rows_grow_and_are_written(dtype, width, page, layout):
    import paper_1804_10112_amd as spt
    host = HostCache([0, 5, 16, 33], page, 3, width, dtype, layers=2, spare=70, room=30, poison=False)
    cache = host.device(layout)
    gen = torch.Generator().manual_seed(1)
    for add in ([1, 1, 1, 1], [0, 16, 3, 0], [7, 0, 0, 9]):
        _extend(host, cache, add, f"extend {add}")
        first = offsets(add)
        for layer in range(2):
            k, v = (torch.randn(first[-1] + 3, 3, width, generator=gen).to(DTYPES[dtype]) for _ in range(2))
            spt.spt_cache_write(cache, layer, i32(first), k.cuda(), v.cuda())
            host.write(layer, first, k, v)
        host.assert_same(cache, f"write {add}")


def test_strides_of_written_tokens():
    import paper_1804_10112_amd as spt
    host = HostCache([9, 20], 8, 2, 64, "bf16", poison=False)
    cache = host.device()
    packed = torch.randn(7, 2, 3, 64, device="cuda").bfloat16()       # k and v as parts of one tensor
    k, v = packed[:, :, 0], packed[:, :, 2]
    spt.spt_cache_write(cache, 0, i32([0, 4, 7]), k, v)
    host.write(0, [0, 4, 7], k.cpu(), v.cpu())
    host.assert_same(cache)


def test_written_tokens_without_a_place_are_left_out():
    """More tokens than the row holds, pages outside the pool, tokens behind the last row."""
    import paper_1804_10112_amd as spt
    host = HostCache([2, 40, 30], 8, 1, 64, "f32", poison=False)
    cache = host.device()
    cache.table[1, 4], cache.table[2, 3] = -1, 12345
    k = torch.randn(30, 1, 64)
    spt.spt_cache_write(cache, 0, i32([0, 5, 9, 12]), k.cuda(), k.cuda())
    K, table = host.K.clone(), host.table
    K[0, table[0][0], 0:2, 0] = k[3:5, 0]                              # the last two of five
    torch.cuda.synchronize()
    assert torch.equal(cache.K.cpu(), K)                               # rows 1 and 2 end in pages that are not there


@pytest.mark.parametrize("pages,rows", [(5, 3), (2000, 40), (5000, 1500), (70_000, 300), (1_300_000, 9)])
def test_pages_are_taken_in_ascending_order(pages, rows):
    """Free pages anywhere in pools of one stretch to many, rows of one block to several."""
    rng = np.random.default_rng(pages)
    host = HostCache([0] * rows, 2, 1, 8, "f32", spare=1, room=8, poison=False)
    host.K = host.V = torch.zeros(1, pages, 2, 1, 8)
    host.refs = (rng.random(pages) < 0.7).astype(int).tolist()
    cache = host.device()
    _extend(host, cache, rng.integers(-1, 9, rows).tolist(), "first")
    _extend(host, cache, rng.integers(0, 7, rows).tolist(), "second")


@pytest.mark.parametrize("free", [0, 1, 3, 4, 9])
def test_rows_are_refused_when_pages_run_out(free):
    host = HostCache([3, 4, 0, 8, 5, 1], 4, 1, 8, "f32", spare=free, room=3, poison=False)
    cache = host.device()
    _extend(host, cache, [1, 5, 4, 0, 9, 2], "rows in order")
    _extend(host, cache, [0, 0, 0, 0, 0, 1], "a row that needs no page")


def test_rows_are_refused_when_the_table_is_full():
    host = HostCache([3, 4, 8], 4, 1, 8, "f32", spare=20, room=1, poison=False)
    cache = host.device()
    _extend(host, cache, [9, 9, 5], "one too long")
    _extend(host, cache, [2 ** 31 - 1, 1, -2 ** 31], "numbers at the ends of int32")


@pytest.mark.parametrize("layout", ["slots", "heads"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [0, 1, 7, 8, 21, 24])
def test_forks_share_pages_and_copy_the_last_one_when_written(length, layout, dtype):
    import paper_1804_10112_amd as spt
    host = HostCache([length, 5, 0, 9, 0], 8, 2, 24, dtype, layers=3, spare=20, room=4, seed=length)
    cache = host.device(layout)
    parents, children = [0, 0, 1], [2, 3, 4]                           # row 3 held something before
    spt.spt_cache_fork(cache, i32(parents), i32(children))
    host.fork(parents, children)
    host.assert_same(cache, "fork")
    _extend(host, cache, [0, 0, 2, 1, 1], "the children go on")
    _extend(host, cache, [1, 1, 0, 0, 0], "then the parents, alone again")
    spt.spt_cache_fork(cache, i32([2, 2]), i32([0, 3]))
    host.fork([2, 2], [0, 3])
    _extend(host, cache, [1, 0, 1, 9, 0], "all who share at once")
    spt.spt_cache_free(cache, i32([0] * 5))
    host.free([0] * 5)
    host.assert_same(cache, "all given back")
    assert not any(host.refs)


def test_forks_that_are_skipped():
    import paper_1804_10112_amd as spt
    host = HostCache([9, 5, 3, 0, 0, 0, 2], 4, 1, 8, "f32", spare=3)
    cache = host.device()
    parents = [0, 1, 2, 7, 0, -1, 0, 1, 6]
    children = [3, 3, 1, 4, 9, 5, -2, 4, 6]        # 3 twice, 1 a parent, rows that are not there, 6 its own child
    spt.spt_cache_fork(cache, i32(parents), i32(children))
    host.fork(parents, children)
    host.assert_same(cache)
    assert host.len[3] == 5 and host.len[1] == 5 and host.len[4] == 5 and host.len[5] == 0


def test_rows_are_cut_and_freed():
    import paper_1804_10112_amd as spt
    host = HostCache([0, 1, 16, 17, 300, 40, 12], 4, 1, 8, "f32")
    cache = host.device()
    for new_len in ([5, 1, 16, 16, 100, -1, 0], [0, 0, 15, 2 ** 31 - 1, 1, 39, -2 ** 31], [0] * 7, [0] * 7):
        spt.spt_cache_free(cache, i32(new_len))
        host.free(new_len)
        host.assert_same(cache, str(new_len))


@pytest.mark.parametrize("dtype,width,page", [("bf16", 64, 16), ("f32", 40, 1), ("f16", 128, 4), ("bf16", 256, 64)])
@pytest.mark.parametrize("layout", ["slots", "heads"])
def test_kept_tokens_are_drawn_together(dtype, width, page, layout):
    import paper_1804_10112_amd as spt
    rng = np.random.default_rng(width)
    counts = [5, 0, 33, 1, 12, 7, 40]
    host = HostCache([n + c for n, c in zip(counts, [0, 9, 50, 3, 1, 16, 3])], page, 3, width, dtype, layers=2, seed=1)
    cache = host.device(layout)
    keep = [[0, 1, 2], [], sorted(rng.permutation(33)[:20].tolist()), [0], [], [6], list(range(1, 40))]
    spt.spt_cache_compact(cache, i32(offsets(counts)), pattern(keep))
    host.compact(offsets(counts), keep)
    host.assert_same(cache)


def test_kept_tokens_of_rows_that_are_too_short_or_lists_out_of_range():
    import paper_1804_10112_amd as spt
    host = HostCache([2, 10], 4, 1, 8, "f32", poison=False)
    cache = host.device()
    keep = spt.DeviceCSR(i32([0, 1, 4]), i32([0, 1, 70, -3]), 5, ordered=True, unique=True)
    spt.spt_cache_compact(cache, i32([0, 4, 8]), keep)                # row 0 has 2 tokens, not 4
    host.len, K = [2, 10], host.K
    p0, p1 = host.slot(1, 6), host.slot(1, 7)
    K[:, p0[0], p0[1]], host.V[:, p0[0], p0[1]] = K[:, p1[0], p1[1]].clone(), host.V[:, p1[0], p1[1]].clone()
    host.cut(1, 9)
    host.assert_same(cache)


def test_a_round_in_a_captured_graph():
    """Extend, write, compact, free and fork as one graph; replays, with eager work between them, follow the host model."""
    import paper_1804_10112_amd as spt
    host = HostCache([5, 30, 0], 4, 2, 64, "bf16", spare=60, room=40, poison=False, layers=2)
    cache = host.device()
    add, refused, ws = i32([6, 6, 0]), i32([0]), cache.workspace(spt.SPT_CACHE_EXTEND)
    first, keep_rows = [0, 6, 12, 12], [[0, 2, 5], [1, 3], []]
    first_dev, keep = i32(first), pattern(keep_rows)
    k, v = (torch.randn(2, 12, 2, 64).bfloat16() for _ in range(2))
    kd, vd = k.cuda(), v.cuda()
    parents, children, cut = i32([1]), i32([2]), i32([-1, 33, -1])

    def device_round():
        spt.spt_cache_extend(cache, add, refused, ws)
        for layer in range(2):
            spt.spt_cache_write(cache, layer, first_dev, kd[layer], vd[layer])
        spt.spt_cache_compact(cache, first_dev, keep)
        spt.spt_cache_free(cache, cut)
        spt.spt_cache_fork(cache, parents, children)

    def host_round():
        assert host.extend([6, 6, 0]) == 0
        for layer in range(2):
            host.write(layer, first, k[layer], v[layer])
        host.compact(first, keep_rows)
        host.free([-1, 33, -1])
        host.fork([1], [2])

    device_round()
    host_round()
    host.assert_same(cache, "eager")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        device_round()
    for step in range(4):
        ws.fill_(170)
        torch.cuda.synchronize()
        g.replay()
        host_round()
        host.assert_same(cache, f"replay {step}")
        assert int(refused.item()) == 0


def test_offsets_beyond_32_bits():
    import paper_1804_10112_amd as spt
    host = HostCache([20, 6], 4, 1, 8, "f32", layers=2, spare=6, poison=False)
    near = host.device()
    pages, page_stride = host.K.shape[1], 2 ** 27                      # 512 MB
    pool = torch.zeros(page_stride * pages * 2, dtype=torch.float32, device="cuda")
    K, V = (torch.as_strided(pool, host.K.shape, (page_stride * pages, page_stride, 8, 8, 1), off) for off in (0, 2 ** 20))
    K.copy_(near.K), V.copy_(near.V)
    cache = spt.DeviceCache(K, V, near.table, near.len, near.refs)
    _extend(host, cache, [7, 2], "extend")
    k = torch.randn(9, 1, 8)
    spt.spt_cache_write(cache, 1, i32([0, 7, 9]), k.cuda(), k.cuda())
    host.write(1, [0, 7, 9], k, k)
    spt.spt_cache_compact(cache, i32([0, 7, 9]), pattern([[1, 4, 6], [1]]))
    host.compact([0, 7, 9], [[1, 4, 6], [1]])
    host.assert_same(cache, "far pages")


def test_caches_of_no_rows_or_no_pages():
    import paper_1804_10112_amd as spt
    empty = spt.DeviceCache(torch.zeros(1, 0, 4, 1, 8, device="cuda"), torch.zeros(1, 0, 4, 1, 8, device="cuda"),
                            torch.full((2, 3), -1, dtype=torch.int32, device="cuda"), i32([0, 0]), i32([]))
    refused = i32([-1])
    spt.spt_cache_extend(empty, i32([1, 0]), refused, empty.workspace(spt.SPT_CACHE_EXTEND))
    assert int(refused.item()) == 1 and empty.len.tolist() == [0, 0]
    k = torch.zeros(1, 1, 8, device="cuda")
    spt.spt_cache_write(empty, 0, i32([0, 1, 1]), k, k)
    spt.spt_cache_free(empty, i32([0, 0]))
    none = spt.DeviceCache(torch.zeros(1, 3, 4, 1, 8, device="cuda"), torch.zeros(1, 3, 4, 1, 8, device="cuda"),
                           torch.zeros(0, 3, dtype=torch.int32, device="cuda"), i32([]), i32([0, 0, 0]))
    refused.fill_(-1)
    spt.spt_cache_extend(none, i32([]), refused, none.workspace(spt.SPT_CACHE_EXTEND))
    assert int(refused.item()) == 0
