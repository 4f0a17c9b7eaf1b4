"""CPU-only checks of the entry points of caches, attention and logits: struct layouts, refusals, workspace sizes."""
import ctypes as C
import os
import subprocess

import pytest

import paper_1804_10112_amd as spt
from paper_1804_10112_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # 256-byte aligned, never read on the host


def _cache(**changes):
    c = B.SptCache()
    for name, value in dict(dtype=B.SPT_BF16, layers=2, heads=4, width=64, page=16, rows=3, row_pages=10, pages=40, layer_stride=163840,
                            page_stride=4096, slot_stride=256, head_stride=64, K=FAKE, V=FAKE, table=FAKE, len=FAKE, refs=FAKE).items():
        setattr(c, name, changes.get(name, value))
    return c


def _csr(rows, cols=8, entries=5, flags=3, dtype=0, vals=FAKE):
    t = B.SptTensor()
    t.order = t.nlevels = 2
    t.dtype = dtype
    t.level[0].kind, t.level[0].mode, t.level[0].N = 0, 0, rows
    o = t.level[1]
    o.kind, o.mode, o.N, o.M, o.flags, o.pos, o.crd = 1, 1, cols, rows, flags, FAKE, FAKE
    t.vals, t.nvals = vals, entries
    return t


def _addr(x):
    return None if x is None else C.addressof(x) if isinstance(x, C.Structure) else x


def test_struct_layouts_match_the_header(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "spt.h"\n'
                   'int main(void) { printf("%zu %zu %zu %zu %zu %zu %d %d\\n", sizeof(spt_cache), offsetof(spt_cache, pages), '
                   'offsetof(spt_cache, refs), sizeof(spt_logit_rules), offsetof(spt_logit_rules, bias), '
                   'offsetof(spt_logit_rules, allowed_stride), SPT_BF16, SPT_CACHE_ATTENTION); return 0; }\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(t) for t in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(B.SptCache), B.SptCache.pages.offset, B.SptCache.refs.offset, C.sizeof(B.SptLogitRules),
                   B.SptLogitRules.bias.offset, B.SptLogitRules.allowed_stride.offset, B.SPT_BF16, B.SPT_CACHE_ATTENTION]


BAD_CACHES = [
    (dict(dtype=B.SPT_F64), 2), (dict(dtype=9), 1), (dict(dtype=-1), 1), (dict(layers=0), 1), (dict(heads=0), 1),
    (dict(heads=70000), 1), (dict(width=0), 2), (dict(width=60), 2), (dict(width=264), 2), (dict(width=-8), 2), (dict(page=0), 2),
    (dict(page=24), 2), (dict(page=1 << 17), 2), (dict(rows=-1), 1), (dict(row_pages=-1), 1), (dict(pages=-1), 1),
    (dict(pages=2 ** 31 - 1), 1), (dict(rows=(1 << 20) + 1, row_pages=1), 2), (dict(rows=1 << 20, row_pages=1 << 11), 2),
    (dict(row_pages=1 << 27), 2), (dict(slot_stride=-256), 1), (dict(head_stride=60), 1), (dict(page_stride=4), 1),
    (dict(layer_stride=1 << 41), 1), (dict(page_stride=1 << 33), 2), (dict(layers=65536, heads=2), 2), (dict(K=None), 1), (dict(V=None), 1), (dict(refs=None), 1), (dict(table=None), 1),
    (dict(len=None), 1), (dict(K=FAKE + 8), 1), (dict(V=FAKE + 2), 1), (dict(dtype=B.SPT_F32, head_stride=62), 1),
]


@pytest.mark.parametrize("changes,status", BAD_CACHES, ids=[str(c[0]) for c in BAD_CACHES])
def test_caches_that_are_refused_by_every_entry_point(changes, status):
    c, lib = _cache(**changes), spt.lib()
    p = C.addressof(c)
    keep, ws = _csr(3), FAKE
    calls = [lib.spt_cache_extend(p, FAKE, FAKE, ws, 1 << 20, None), lib.spt_cache_free(p, FAKE, None),
             lib.spt_cache_fork(p, 1, FAKE, FAKE, None), lib.spt_cache_write(p, 0, FAKE, 1, FAKE, FAKE, 256, 64, None),
             lib.spt_cache_compact(p, FAKE, C.addressof(keep), None),
             lib.spt_cache_attention(p, 0, FAKE, 1, None, FAKE, 4, 256, 64, 1.0, FAKE, 256, 64, None, ws, 1 << 40, None)]
    assert calls == [status] * len(calls) and spt.spt_last_error()
    assert lib.spt_cache_workspace_bytes(B.SPT_CACHE_EXTEND, p, 0) == 0


def test_a_null_cache_is_refused():
    lib = spt.lib()
    assert lib.spt_cache_extend(None, FAKE, FAKE, FAKE, 1 << 20, None) == 1
    assert lib.spt_cache_workspace_bytes(B.SPT_CACHE_ATTENTION, None, 4) == 0


def test_workspaces():
    lib, c = spt.lib(), _cache()
    p = C.addressof(c)
    assert lib.spt_cache_workspace_bytes(B.SPT_CACHE_EXTEND, p, 0) >= 256
    assert lib.spt_cache_workspace_bytes(B.SPT_CACHE_ATTENTION, p, 8) >= 256
    for q_heads in (0, -4, 6, 65540):
        assert lib.spt_cache_workspace_bytes(B.SPT_CACHE_ATTENTION, p, q_heads) == 0 and "q_heads" in spt.spt_last_error()
    assert lib.spt_cache_workspace_bytes(7, p, 8) == 0 and "op" in spt.spt_last_error()
    need = lib.spt_cache_workspace_bytes(B.SPT_CACHE_EXTEND, p, 0)
    assert lib.spt_cache_extend(p, FAKE, FAKE, None, 0, None) == B.SPT_ERR_WORKSPACE
    assert lib.spt_cache_extend(p, FAKE, FAKE, FAKE, need - 256, None) == B.SPT_ERR_WORKSPACE
    assert lib.spt_cache_extend(p, FAKE, FAKE, FAKE + 128, need, None) == 1
    need = lib.spt_cache_workspace_bytes(B.SPT_CACHE_ATTENTION, p, 8)
    call = lambda ws, n: lib.spt_cache_attention(p, 0, FAKE, 1, None, FAKE, 8, 512, 64, 1.0, FAKE, 512, 64, None, ws, n, None)
    assert call(FAKE, need - 1) == B.SPT_ERR_WORKSPACE and call(None, need) == B.SPT_ERR_WORKSPACE and call(FAKE + 16, need) == 1


def test_refusals_of_extend_free_fork():
    lib, c = spt.lib(), _cache()
    p = C.addressof(c)
    assert lib.spt_cache_extend(p, None, FAKE, FAKE, 1 << 20, None) == 1
    assert lib.spt_cache_extend(p, FAKE, None, FAKE, 1 << 20, None) == 1
    assert lib.spt_cache_free(p, None, None) == 1
    assert lib.spt_cache_fork(p, -1, FAKE, FAKE, None) == 1
    assert lib.spt_cache_fork(p, 65537, FAKE, FAKE, None) == 2
    assert lib.spt_cache_fork(p, 2, None, FAKE, None) == 1 and lib.spt_cache_fork(p, 2, FAKE, None, None) == 1
    assert lib.spt_cache_fork(p, 0, None, None, None) == 0


def test_refusals_of_write():
    lib, c = spt.lib(), _cache()
    call = lambda layer=0, first=FAKE, T=4, k=FAKE, v=FAKE, ts=256, hs=64: lib.spt_cache_write(
        C.addressof(c), layer, first, T, k, v, ts, hs, None)
    assert [call(layer=2), call(layer=-1), call(T=-1), call(first=None), call(k=None), call(v=None), call(k=FAKE + 8), call(v=FAKE + 4),
            call(ts=-256), call(hs=63), call(ts=1 << 40)] == [1] * 11
    assert call(T=(1 << 24) + 1) == 2 and call(T=0, k=None) == 0


def test_refusals_of_compact():
    lib, c = spt.lib(), _cache()
    call = lambda keep, first=FAKE: lib.spt_cache_compact(C.addressof(c), first, _addr(keep), None)
    assert call(None) == 1 and call(_csr(4)) == 1 and call(_csr(3), first=None) == 1
    assert call(_csr(3, flags=1)) == 2 and call(_csr(3, flags=2)) == 2
    coo = _csr(3)
    coo.level[1].kind = 2
    assert call(coo) != 0
    negative = _csr(3)
    negative.nvals = -1
    assert call(negative) == 1
    no_pos = _csr(3)
    no_pos.level[1].pos = None
    assert call(no_pos) == 1


def test_refusals_of_attention():
    lib, c = spt.lib(), _cache()
    need = lib.spt_cache_workspace_bytes(B.SPT_CACHE_ATTENTION, C.addressof(c), 8)

    def call(layer=0, first=FAKE, T=5, tree=None, q=FAKE, heads=8, qt=512, qh=64, out=FAKE, ot=512, oh=64):
        return lib.spt_cache_attention(C.addressof(c), layer, first, T, _addr(tree), q, heads, qt, qh, 1.0, out, ot, oh, None, FAKE,
                                       need, None)

    assert [call(layer=2), call(T=-1), call(first=None), call(q=None), call(out=None), call(heads=6), call(heads=0), call(q=FAKE + 2),
            call(out=FAKE + 8), call(qt=-8), call(qh=3), call(ot=7), call(oh=-64), call(tree=_csr(4)), call(tree=_csr(6))] == [1] * 15
    assert call(T=(1 << 24) + 1) == 2 and call(T=1 << 24, heads=4 * 1024) == 2
    csc = _csr(5)
    csc.level[0].mode, csc.level[1].mode = 1, 0
    assert call(tree=csc) == 2
    assert call(T=0, q=None) == 0


def test_refusals_of_logits():
    lib = spt.lib()

    def call(dtype=B.SPT_F16, R=3, V=100, logits=FAKE, stride=104, out=FAKE, out_stride=104, rules=True, **given):
        r = B.SptLogitRules()
        r.first, r.sequences = FAKE, 2
        for name, value in given.items():
            setattr(r, name, _addr(value))
        return lib.spt_adjust_logits(dtype, R, V, logits, stride, C.addressof(r) if rules else None, out, out_stride, None)

    assert call(dtype=B.SPT_F64) == 2 and call(dtype=5) == 1 and call(rules=False) == 1
    assert [call(R=-1), call(V=-1), call(V=2 ** 31 - 1), call(sequences=-1), call(first=None), call(stride=99), call(out_stride=99),
            call(logits=None), call(out=None), call(logits=FAKE + 1), call(dtype=B.SPT_F32, out=FAKE + 2), call(out_stride=108)] == [1] * 12
    assert call(R=(1 << 24) + 1) == 2 and call(V=(1 << 27) + 1, stride=1 << 28, out_stride=1 << 28) == 2
    assert call(seen=_csr(3)) == 1 and call(tree=_csr(3)) == 1 and call(tree=_csr(2), drafts=FAKE) == 1
    assert call(bias=_csr(3)) == 1 and call(bias=_csr(2, dtype=1)) == 2 and call(bias=_csr(2, flags=1)) == 2
    assert call(bias=_csr(2, vals=None)) == 1
    assert call(allowed=FAKE, allowed_stride=3) == 1
    assert call(R=0, logits=None) == 0 and call(V=0, logits=None) == 0


def test_the_binding_refuses_tensors_that_do_not_fit():
    import torch
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32)
    make = lambda K=z(1, 4, 16, 2, 64), V=z(1, 4, 16, 2, 64), table=i32(0, 0, 0, 0).view(2, 2), length=i32(0, 0), refs=i32(0, 0, 0, 0): \
        spt.DeviceCache(K, V, table, length, refs)
    cache = make()
    for bad in (dict(V=z(1, 4, 16, 2, 32)), dict(K=z(4, 16, 2, 64)), dict(refs=i32(0)), dict(length=i32(0)), dict(table=i32(0, 0)),
                dict(V=z(1, 4, 16, 2, 64, dtype=torch.float16)), dict(refs=torch.zeros(4, dtype=torch.int64)),
                dict(V=z(1, 4, 2, 16, 64).transpose(2, 3))):
        with pytest.raises(spt.SptError):
            make(**bad)
    q, first = z(3, 4, 64), i32(0, 1, 3)
    for bad in (dict(q=z(3, 4, 32)), dict(out=z(2, 4, 64)), dict(out=z(3, 2, 64)), dict(q=z(3, 4, 64, dtype=torch.float32)),
                dict(first=i32(0, 1)), dict(lse=z(3, 4)), dict(q=z(3, 64, 4).transpose(1, 2)), dict(q=z(4, 64))):
        args = dict(q=q, out=z(3, 4, 64), first=first, lse=None)
        args.update(bad)
        with pytest.raises(spt.SptError):
            spt.spt_cache_attention(cache, 0, args["first"], None, args["q"], 1.0, args["out"], args["lse"])
    with pytest.raises(spt.SptError):
        spt.spt_cache_write(cache, 0, first, z(3, 2, 64), z(2, 2, 64))
    with pytest.raises(spt.SptError):
        spt.spt_cache_extend(cache, i32(1), i32(0), None)
    with pytest.raises(spt.SptError):
        spt.spt_cache_fork(cache, i32(0), i32(0, 1))
    with pytest.raises(spt.SptError):
        spt.LogitRules()
    with pytest.raises(spt.SptError):
        spt.spt_adjust_logits(z(2, 8), spt.LogitRules(first=first), z(2, 9))
    with pytest.raises(TypeError):
        spt.spt_adjust_logits(torch.zeros(2, 8, dtype=torch.int32), spt.LogitRules(first=first), torch.zeros(2, 8, dtype=torch.int32))
