"""The operators together, as a server of drafted tokens runs them: room is made, drafts are written and attended to in every layer, their
logits are changed by the rules, the accepted ones kept, rows forked and freed. Against the host model and float64, step by step."""
import numpy as np
import pytest
import torch

from cache_util import HostCache, assert_within, attention_reference, offsets, pattern, random_q, random_tree

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")


def test_steps_of_drafting_with_forks():
    import paper_1804_10112_amd as spt
    rng = np.random.default_rng(3)
    layers, heads, q_heads, width, V = 2, 2, 8, 64, 3000
    host = HostCache([37, 8, 0, 0, 90], 16, heads, width, "bf16", layers=layers, spare=60, room=12, seed=3)
    cache = host.device("heads")
    refused, extend_ws = i32([0]), cache.workspace(spt.SPT_CACHE_EXTEND)
    ws = cache.workspace(spt.SPT_CACHE_ATTENTION, q_heads)
    history = [rng.integers(0, V, n).tolist() for n in host.len]
    for step in range(5):
        if step == 1:                                  # two answers to the prompt of row 0, a row for each
            spt.spt_cache_fork(cache, i32([0, 0]), i32([2, 3]))
            host.fork([0, 0], [2, 3])
            history[2], history[3] = list(history[0]), list(history[0])
        counts = [int(n) if host.len[s] else 0 for s, n in enumerate(rng.integers(1, 14, 5))]
        first, tree = offsets(counts), random_tree(counts, step)
        T = first[-1]
        spt.spt_cache_extend(cache, i32(counts), refused, extend_ws)
        assert host.extend(counts) == 0
        first_dev, tree_dev = i32(first), pattern(tree)
        out, lse = torch.empty(T, q_heads, width, dtype=torch.bfloat16, device="cuda"), torch.empty(T, q_heads, device="cuda")
        for layer in range(layers):
            k, v = (torch.randn(T, heads, width).bfloat16() for _ in range(2))
            q = random_q(T, q_heads, width, "bf16", 10 * step + layer)
            spt.spt_cache_write(cache, layer, first_dev, k.cuda(), v.cuda())
            spt.spt_cache_attention(cache, layer, first_dev, tree_dev, q.cuda(), 0.125, out, lse, ws)
            host.write(layer, first, k, v)
            ref, ref_lse, bound, lse_bound = attention_reference(host, layer, counts, tree, q, 0.125)
            assert_within(out, ref, bound, f"step {step} layer {layer}")
            assert_within(lse, ref_lse, lse_bound, f"step {step} layer {layer} lse")
        # the rules: what was seen and what lies on a row's way weighs on it
        drafts = rng.integers(0, V, T).tolist()
        logits = torch.randn(T, V)
        seen = spt.DeviceCSR(i32(offsets([len(h) for h in history])), i32([t for h in history for t in h]), V)
        rules = spt.LogitRules(first=first_dev, tree=tree_dev, drafts=i32(drafts), seen=seen,
                               presence=torch.full((5,), 2.0, device="cuda"))
        changed = torch.empty(T, V, device="cuda")
        spt.spt_adjust_logits(logits.cuda(), rules, changed)
        want = logits.clone()
        for s in range(5):
            for r in range(first[s], first[s + 1]):
                want[r, sorted(set(history[s]) | {drafts[first[s] + j] for j in tree[r]})] -= 2.0
        assert torch.equal(changed.cpu(), want), f"step {step} logits"
        # the way to some node is accepted
        keep = [tree[first[s] + int(rng.integers(0, n))] if n else [] for s, n in enumerate(counts)]
        spt.spt_cache_compact(cache, first_dev, pattern(keep))
        host.compact(first, keep)
        for s, kept in enumerate(keep):
            history[s] += [drafts[first[s] + j] for j in kept]
        if step == 3:                                  # an answer has ended, its row is free for another
            spt.spt_cache_free(cache, i32([-1, -1, 0, -1, -1]))
            host.free([-1, -1, 0, -1, -1])
            history[2] = []
        host.assert_same(cache, f"step {step}")
        assert int(refused.item()) == 0 and [len(h) for h in history] == host.len
    spt.spt_cache_free(cache, i32([0] * 5))
    assert not any(cache.refs.tolist())
