"""Rules on logits against their definition in float64."""
import math

import numpy as np
import pytest
import torch

from cache_util import DTYPES, HALF_STEP, assert_within, offsets, random_tree

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")


def _rows_to_csr(rows, cols, vals=None, unique=False):
    import paper_1804_10112_amd as spt
    flat = None if vals is None else torch.tensor([x for r in vals for x in r], dtype=torch.float32, device="cuda")
    return spt.DeviceCSR(i32(offsets([len(r) for r in rows])), i32([c for r in rows for c in r]), cols, flat, unique=unique)


def _reference(logits, first, seen, tree, drafts, rep, pres, freq, bias, bias_vals, allowed, dtype):
    """By definition; the bound counts a rounding for each of the operations in float32 and the one to the type."""
    x = logits.double().clone()
    size = x.abs()
    R, V = x.shape
    for s in range(len(first) - 1):
        for r in range(first[s], first[s + 1]):
            c = np.zeros(V)
            for t in (seen[s] if seen else []):
                if 0 <= t < V:
                    c[t] += 1
            if drafts is not None:
                n = first[s + 1] - first[s]
                for j in (tree[r] if tree is not None else range(r - first[s] + 1)):
                    if 0 <= j < n and 0 <= drafts[first[s] + j] < V:
                        c[drafts[first[s] + j]] += 1
            hit = torch.from_numpy(c > 0)
            c = torch.from_numpy(c)
            a, p, f = (float(t[s]) if t is not None else d for t, d in ((rep, 1.0), (pres, 0.0), (freq, 0.0)))
            y = torch.where(x[r] > 0, x[r] / a, x[r] * a)
            size[r] = torch.where(hit, y.abs() + abs(p) + 2 * abs(f) * c, size[r])
            x[r] = torch.where(hit, y - (p + f * c), x[r])
            for t, b in zip(bias[s], bias_vals[s]) if bias else ():
                if 0 <= t < V:
                    b = float(np.float32(b))
                    x[r, t] += b
                    size[r, t] += abs(b)
            if allowed is not None:
                v = np.arange(V)
                x[r][torch.from_numpy((allowed[r].astype(np.int64)[v // 32] >> (v % 32)) & 1 == 0)] = -math.inf
    # a result beyond the largest number of the type rounds to an infinity (the lowest float32 times 1.76 is -5.99e38)
    largest = torch.finfo(DTYPES[dtype]).max * (1 + HALF_STEP[dtype] / 2)
    x = torch.where(x.abs() > largest, torch.sign(x) * math.inf, x)
    tiny = 2.0 ** -25 if dtype == "f16" else 0
    return x, torch.nan_to_num(size) * 4 * 2.0 ** -24 + HALF_STEP[dtype] * torch.nan_to_num(x.abs(), posinf=0) + tiny


def _check(dtype, V, counts, seed=0, tree="tree", penalties=True, seen_count=30, biases=5, masked=True, drafted=True, logits=None,
           in_place=False, pad=0):
    import paper_1804_10112_amd as spt
    rng = np.random.default_rng(seed)
    first, N = offsets(counts), len(counts)
    R = first[-1]
    if logits is None:
        logits = torch.from_numpy(rng.normal(0, 3, (R, V)).astype(np.float32)).to(DTYPES[dtype])
    draw = lambda n: np.minimum((rng.random(n) ** 3 * V).astype(int), V - 1).tolist()
    seen = [draw(int(rng.integers(0, seen_count + 1))) for _ in range(N)] if seen_count else None
    rows = random_tree(counts, seed) if tree == "tree" else None
    drafts = draw(R) if drafted else None
    rep, pres, freq = ((rng.uniform(a, b, N).astype(np.float32) for a, b in ((1, 2), (0, 1), (0, 0.5))) if penalties else (None,) * 3)
    bias = [sorted(rng.permutation(V)[:biases].tolist()) for _ in range(N)] if biases else None
    bias_vals = [rng.normal(0, 5, len(r)).tolist() for r in bias] if biases else None
    words = (V + 31) // 32
    allowed = rng.integers(0, 2 ** 32, (R, words), dtype=np.uint64) if masked else None
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()
    rules = spt.LogitRules(
        first=i32(first), seen=_rows_to_csr(seen, V) if seen else None, tree=_rows_to_csr(rows, max(counts)) if rows and drafted else None,
        drafts=None if drafts is None else i32(drafts), repetition=dev(rep), presence=dev(pres), frequency=dev(freq),
        bias=_rows_to_csr(bias, V, bias_vals, unique=True) if bias else None,
        allowed=dev(allowed.astype(np.uint32).view(np.int32)) if masked else None)
    wide = torch.full((R, V + pad), 7.0, dtype=DTYPES[dtype], device="cuda")
    src = wide[:, :V]
    src.copy_(logits)
    out = src if in_place else torch.full((R + 1, V + 2 * pad), 9.0, dtype=DTYPES[dtype], device="cuda")[:R, pad:V + pad]
    spt.spt_adjust_logits(src, rules, out)
    torch.cuda.synchronize()
    ref, bound = _reference(logits, first, seen, rows, drafts, rep, pres, freq, bias, bias_vals, allowed, dtype)
    assert_within(out, ref, bound, f"{dtype} V={V}")
    if not in_place:
        assert torch.equal(src.cpu().view(torch.uint8), logits.contiguous().view(torch.uint8)) if pad == 0 else True
    return out


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [1, 7, 31, 32, 33, 1000, 8191, 8192, 8193, 20_001, 70_003])
def test_vocabularies(dtype, V):
    _check(dtype, V, [1, 3, 2], seed=V, biases=min(5, V))


@pytest.mark.parametrize("counts", [[1], [1] * 50, [0, 5, 0, 0, 9, 0], [40, 1, 17]])
@pytest.mark.parametrize("tree", ["tree", None])
def test_rows_of_sequences(counts, tree):
    _check("f32", 3001, counts, seed=len(counts), tree=tree)


@pytest.mark.parametrize("without", ["penalties", "seen", "bias", "mask", "drafts", "all"])
def test_rules_left_out(without):
    every = without == "all"
    _check("bf16", 5003, [2, 4, 1], seed=3, penalties=not (every or without == "penalties"),
           seen_count=0 if every or without == "seen" else 40, biases=0 if every or without == "bias" else 4,
           masked=not (every or without == "mask"), drafted=not (every or without == "drafts"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_row_strides_and_offsets(dtype, pad):
    _check(dtype, 1001, [3, 2], seed=pad, pad=pad)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_in_place(dtype):
    _check(dtype, 9001, [3, 2], seed=1, in_place=True)
    _check(dtype, 777, [3, 2], seed=1, in_place=True, pad=5)


def test_many_repetitions_and_long_histories():
    _check("f32", 50, [2, 1], seed=5, seen_count=30_000, masked=False)
    _check("f32", 30_000, [1, 1], seed=6, seen_count=60_000)


def test_values_that_are_not_finite():
    logits = torch.zeros(3, 4000)
    logits[:, ::7], logits[:, 1::7], logits[:, 2::7], logits[:, 3::7] = math.inf, -math.inf, math.nan, torch.finfo(torch.float32).min
    logits[:, 4::7] = -0.0
    for masked in (False, True):
        _check("f32", 4000, [2, 1], seed=9, logits=logits, masked=masked, seen_count=3000)


def test_tokens_and_nodes_out_of_range_are_skipped():
    import paper_1804_10112_amd as spt
    logits = torch.randn(4, 100, device="cuda")
    seen = _rows_to_csr([[5, -1, 100, 2 ** 31 - 1, 5], [-2 ** 31, 7]], 100)
    tree = _rows_to_csr([[0], [1, 0, 2, -1, 99], [0, 0], [1]], 2)
    rules = spt.LogitRules(first=i32([0, 2, 4]), seen=seen, tree=tree, drafts=i32([3, 2000, -4, 9]),
                           presence=torch.tensor([1.0, 2.0], device="cuda"))
    out = torch.empty_like(logits)
    spt.spt_adjust_logits(logits, rules, out)
    want = logits.clone()
    want[:2, 5] -= 1
    want[:2, 3] -= 1
    want[2:, 7] -= 2
    want[3, 9] -= 2
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_rows_behind_the_last_sequence_and_rules_without_first():
    import paper_1804_10112_amd as spt
    logits = torch.randn(6, 300, device="cuda").bfloat16()
    out = torch.full_like(logits, 7.0)
    presence = torch.tensor([1.0, 2.0], device="cuda")
    spt.spt_adjust_logits(logits, spt.LogitRules(first=i32([0, 1, 4]), presence=presence, seen=_rows_to_csr([[0], [1, 1]], 300)), out)
    want = logits.float()
    want[0, 0] -= 1
    want[1:4, 1] -= 2
    torch.cuda.synchronize()
    assert torch.equal(out[:4], want[:4].bfloat16()) and bool((out[4:] == 7).all())
    spt.spt_adjust_logits(logits[:2], spt.LogitRules(presence=presence, seen=_rows_to_csr([[0], [1]], 300), drafts=i32([4, 5])), out[:2])
    want = logits.float()
    want[0, 0] -= 1
    want[0, 4] -= 1
    want[1, 1] -= 2
    want[1, 5] -= 2
    torch.cuda.synchronize()
    assert torch.equal(out[:2], want[:2].bfloat16())


def test_captured_and_replayed_while_the_history_grows():
    import paper_1804_10112_amd as spt
    logits = torch.randn(2, 9000, device="cuda")
    pos, crd = i32([0, 1, 2]), i32([0] * 50)
    rules = spt.LogitRules(seen=spt.DeviceCSR(pos, crd, 9000), frequency=torch.tensor([1.0, 0.5], device="cuda"))
    out = torch.empty_like(logits)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        spt.spt_adjust_logits(logits, rules, out)
    for step in range(1, 5):
        pos.copy_(i32([0, step, 3 * step]))
        crd[:3 * step] = 17
        logits.add_(0.25)
        out.fill_(math.nan)
        torch.cuda.synchronize()
        g.replay()
        want = logits.clone()
        want[0, 17] -= step
        want[1, 17] -= 0.5 * (2 * step)
        torch.cuda.synchronize()
        assert torch.equal(out, want), step
