"""CPU-only checks of what the binding of caches, attention and logits refuses before a kernel is given a pointer."""
import pytest
import torch

import paper_1804_10112_amd as spt

i32 = lambda *a: torch.tensor(a, dtype=torch.int32)


def _words(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


@pytest.mark.parametrize("mask", [_words(1, 100).expand(8, 100), _words(8, 1).expand(8, 100), _words(300).as_strided((8, 100), (20, 1)),
                                  _words(8, 200)[:, ::2], _words(100, 8).t(), _words(8), _words(8, 100).long()],
                         ids=["one row for all", "one word for all", "overlapping rows", "every other word", "words apart", "one axis", "int64"])
def test_masks_whose_rows_lie_otherwise_are_refused(mask):
    """The kernel reads row r at r * stride, so a stride below the words of a row would be read as another one."""
    with pytest.raises(spt.SptError):
        spt.LogitRules(first=i32(0, 8), allowed=mask)


@pytest.mark.parametrize("mask,stride", [(_words(8, 100), 100), (_words(8, 200)[:, 50:150], 200), (_words(1, 100), 100),
                                         (_words(4, 200)[:1, 10:90], 80), (_words(8, 1), 1), (_words(8, 7)[:, 3:4], 7)])
def test_strides_of_masks(mask, stride):
    assert spt.LogitRules(first=i32(0, 8), allowed=mask).c.allowed_stride == stride


def test_a_mask_with_too_few_words_for_the_vocabulary_is_refused():
    """Whatever its stride: the bits behind a row's last word are another tensor's."""
    logits = torch.zeros(8, 321)
    rules = spt.LogitRules(first=i32(0, 8), allowed=_words(8, 200)[:, :10])
    with pytest.raises(spt.SptError, match="words"):
        spt.spt_adjust_logits(logits, rules, torch.empty_like(logits))


# ---- devices: a pointer of another device, or of the host, is an invalid address to the kernel ------------------------------------

class OnDevice:
    """A tensor that says it lies on device `at`: the checks ask for nothing else, and no call here reaches a kernel."""

    def __init__(self, t, at=0):
        self.t, self.at = t, at

    def get_device(self):
        return self.at

    def __getattr__(self, name):
        return getattr(self.t, name)


def _cache(at=0):
    pool = lambda: OnDevice(torch.zeros(1, 4, 16, 2, 64), at)
    ints = lambda *a: OnDevice(i32(*a), at)
    return spt.DeviceCache(pool(), pool(), OnDevice(i32(0, 1, 2, 3).view(2, 2), at), ints(0, 0), ints(0, 0, 0, 0))


@pytest.fixture
def calls(monkeypatch):
    """The names of the entry points that a test gets through to, on a machine whose current device is 0."""
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: reached.append(name) or 0

    real = spt.lib()
    monkeypatch.setattr(spt.binding, "lib", lambda: Library())
    monkeypatch.setattr(spt.binding, "_device", lambda: 0)
    monkeypatch.setattr(spt.binding, "_raw_stream", lambda device: 0)
    yield reached
    assert real is not None


def _arguments(at=0):
    ints = lambda *a: OnDevice(i32(*a), at)
    tokens = lambda heads: OnDevice(torch.zeros(3, heads, 64), at)
    return dict(first=ints(0, 1, 3), ints=ints(0, 0), one=ints(0), k=tokens(2), v=tokens(2), q=tokens(4), out=tokens(4),
                lse=OnDevice(torch.zeros(3, 4), at), ws=OnDevice(torch.zeros(256, dtype=torch.uint8), at),
                tree=spt.DeviceCSR(ints(0, 1, 2, 3), ints(0, 0, 1), 2), keep=spt.DeviceCSR(ints(0, 1, 2), ints(0, 1), 2, None, True, True),
                logits=OnDevice(torch.zeros(3, 8), at), changed=OnDevice(torch.zeros(3, 8), at),
                rules=spt.LogitRules(first=ints(0, 1, 3), drafts=ints(1, 2, 3)))


ENTRIES = {
    "extend": (lambda c, a: spt.spt_cache_extend(c, a["ints"], a["one"], a["ws"]), ("ints", "one", "ws")),
    "write": (lambda c, a: spt.spt_cache_write(c, 0, a["first"], a["k"], a["v"]), ("first", "k", "v")),
    "compact": (lambda c, a: spt.spt_cache_compact(c, a["first"], a["keep"]), ("first", "keep")),
    "free": (lambda c, a: spt.spt_cache_free(c, a["ints"]), ("ints",)),
    "fork": (lambda c, a: spt.spt_cache_fork(c, a["ints"], a["one"]), ("ints", "one")),
    "attention": (lambda c, a: spt.spt_cache_attention(c, 0, a["first"], a["tree"], a["q"], 1.0, a["out"], a["lse"], a["ws"]),
                  ("first", "tree", "q", "out", "lse", "ws")),
    "adjust_logits": (lambda c, a: spt.spt_adjust_logits(a["logits"], a["rules"], a["changed"]), ("logits", "rules", "changed")),
}


@pytest.mark.parametrize("entry", ENTRIES)
@pytest.mark.parametrize("elsewhere", [1, -1])
def test_tensors_of_another_device_or_of_the_host_are_refused(calls, entry, elsewhere):
    call, names = ENTRIES[entry]
    call(_cache(), _arguments())
    assert len(calls) == 1
    for name in names:
        with pytest.raises(spt.SptError):
            call(_cache(), {**_arguments(), name: _arguments(elsewhere)[name]})
    assert len(calls) == 1


@pytest.mark.parametrize("entry", ENTRIES)
@pytest.mark.parametrize("where", [1, -1])
def test_calls_that_lie_on_another_device_than_the_current_one_or_on_the_host_are_refused(calls, entry, where):
    with pytest.raises(spt.SptError):
        ENTRIES[entry][0](_cache(where), _arguments(where))
    assert not calls


@pytest.mark.parametrize("entry", ENTRIES)
def test_the_first_call_of_a_process_is_checked_too(calls, monkeypatch, entry):
    """Which device is current is asked even when no call has asked for it before."""
    monkeypatch.setattr(spt.binding, "_device", None)
    monkeypatch.setattr(spt.binding, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: type("Stream", (), {"cuda_stream": 0})())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    with pytest.raises(spt.SptError):
        ENTRIES[entry][0](_cache(1), _arguments(1))
    assert not calls


def test_streams_of_another_device_are_refused(calls):
    stream = lambda device: type("Stream", (), {"cuda_stream": 64, "device_index": device})()
    spt.spt_cache_free(_cache(), _arguments()["ints"], stream=stream(0))
    spt.spt_cache_free(_cache(), _arguments()["ints"], stream=64)          # a plain handle says nothing of its device
    with pytest.raises(spt.SptError):
        spt.spt_cache_free(_cache(), _arguments()["ints"], stream=stream(1))
    assert len(calls) == 2


def test_descriptors_of_tensors_on_several_devices_are_refused():
    ints = lambda at, *a: OnDevice(i32(*a), at)
    with pytest.raises(spt.SptError):
        spt.DeviceCSR(ints(0, 0, 1), ints(1, 0), 2)
    with pytest.raises(spt.SptError):
        spt.DeviceCSR(ints(0, 0, 1), ints(0, 0), 2, OnDevice(torch.zeros(1), 1))
    for given in (dict(seen=spt.DeviceCSR(ints(1, 0, 1), ints(1, 0), 2)), dict(presence=OnDevice(torch.zeros(1), 1)),
                  dict(drafts=ints(-1, 0)), dict(allowed=OnDevice(_words(1, 1), 1)),
                  dict(bias=spt.DeviceCSR(ints(-1, 0, 1), ints(-1, 0), 2, OnDevice(torch.zeros(1), -1)))):
        with pytest.raises(spt.SptError):
            spt.LogitRules(first=ints(0, 0, 1), **given)


@pytest.mark.parametrize("scale,status", [(float("nan"), 1), (float("inf"), 1), (-float("inf"), 1), (3e38, 1), (-3e38, 1), (2.0 ** 127, 0),
                                          (-2.0 ** 127, 0), (0.0, 0), (1e-45, 0)])
def test_scales_that_no_score_can_be_multiplied_with_are_refused(scale, status):
    import ctypes
    c = spt.binding.SptCache()
    for name, value in dict(dtype=spt.SPT_BF16, layers=1, heads=2, width=64, page=16, rows=0, row_pages=2, pages=0, layer_stride=0,
                            page_stride=2048, slot_stride=128, head_stride=64).items():
        setattr(c, name, value)
    p, lib = ctypes.addressof(c), spt.lib()
    need = lib.spt_cache_workspace_bytes(spt.SPT_CACHE_ATTENTION, p, 4)
    # no rows: a call that is accepted does nothing
    assert lib.spt_cache_attention(p, 0, None, 0, None, None, 4, 256, 64, scale, None, 256, 64, None, 0x10000, need, None) == status
    assert status == 0 or "scale" in spt.spt_last_error()


def test_strides_of_axes_of_one_do_not_count():
    """torch leaves them as they come: K of a pool with the layers behind the pages, V of one of its own."""
    K, V = torch.zeros(4, 1, 16, 2, 64).transpose(0, 1), torch.zeros(1, 4, 16, 2, 64)
    assert K.stride() != V.stride()
    cache = spt.DeviceCache(K, V, i32(0, 1, 2, 3).view(2, 2), i32(0, 0), i32(0, 0, 0, 0))
    assert (cache.c.layer_stride, cache.c.page_stride, cache.c.slot_stride, cache.c.head_stride) == (0, 2048, 128, 64)
    with pytest.raises(spt.SptError):
        spt.DeviceCache(K.expand(2, -1, -1, -1, -1), V.repeat(2, 1, 1, 1, 1), i32(0, 1, 2, 3).view(2, 2), i32(0, 0), i32(0, 0, 0, 0))
