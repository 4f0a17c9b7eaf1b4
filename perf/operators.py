"""What a server of drafted tokens runs between two steps of its model, as measurable cases: attention of drafted tokens over a
paged cache, the care of that cache's pages, and the rules that change logits before a token is chosen.

A cache holds the keys and values of some sequences in pages: K[l, p, o, h, d] is layer l, page p, slot o of the page, head h,
value d. Row s of `table` lists the pages of sequence s (-1: none), len[s] is the number of its tokens, refs[p] in how many rows
page p is listed; a page of no row is free. The last first[s+1] - first[s] tokens of a sequence are drafted ones. Which of them a
drafted token sees says a CSR pattern (one row for each drafted token, columns counted within its sequence); without a pattern it
sees those before it and itself.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one user, one token: the call's latency
        {"name": "attend_one_token", "op": "attention", "dtype": "bf16", "rows": 1, "shortest": 500, "longest": 500, "drafts": 1,
         "uneven": False, "tree": "causal", "q_heads": 32, "heads": 8, "width": 128, "page": 16, "layout": "slots"},
        # a full batch that decodes token by token: the cache is read once, and that is the time
        {"name": "attend_batch", "op": "attention", "dtype": "bf16", "rows": 64, "shortest": 2000, "longest": 8000, "drafts": 1,
         "uneven": False, "tree": "causal", "q_heads": 32, "heads": 8, "width": 128, "page": 16, "layout": "slots"},
        # a batch that verifies trees of drafted tokens, of other sizes each
        {"name": "attend_tree", "op": "attention", "dtype": "f16", "rows": 16, "shortest": 1000, "longest": 4001, "drafts": 29,
         "uneven": True, "tree": "tree", "q_heads": 32, "heads": 8, "width": 128, "page": 32, "layout": "heads"},
        # one long document and a tree: few rows, so the long axis has to be split
        {"name": "attend_tree_long", "op": "attention", "dtype": "bf16", "rows": 1, "shortest": 100_001, "longest": 100_001,
         "drafts": 16, "uneven": False, "tree": "tree", "q_heads": 16, "heads": 4, "width": 128, "page": 64, "layout": "slots"},
        # a chunk of a prompt behind what is cached of it: the matrix products bound it
        {"name": "attend_chunk", "op": "attention", "dtype": "bf16", "rows": 2, "shortest": 2500, "longest": 4096, "drafts": 1024,
         "uneven": False, "tree": "causal", "q_heads": 32, "heads": 8, "width": 128, "page": 16, "layout": "slots"},
        # 32-bit values, every head with keys of its own, an odd width, patterns that are no trees
        {"name": "attend_f32", "op": "attention", "dtype": "f32", "rows": 8, "shortest": 100, "longest": 1500, "drafts": 7,
         "uneven": True, "tree": "pattern", "q_heads": 12, "heads": 12, "width": 80, "page": 8, "layout": "heads"},
        # a drafting step of one user: pages taken, drafts written, the accepted ones drawn together, pages given back
        {"name": "draft_round_one", "op": "round", "dtype": "f16", "rows": 1, "shortest": 200, "longest": 200, "drafts": 5,
         "uneven": False, "layers": 2, "heads": 8, "width": 64, "page": 16, "layout": "slots"},
        # the same for a batch
        {"name": "draft_round_batch", "op": "round", "dtype": "bf16", "rows": 48, "shortest": 100, "longest": 500, "drafts": 64,
         "uneven": True, "layers": 4, "heads": 8, "width": 128, "page": 16, "layout": "slots"},
        # several answers to each of some prompts: the prompts' pages are shared, and the last one is copied when it is written to
        {"name": "fork_prompts", "op": "fork", "dtype": "bf16", "rows": 60, "parents": 4, "shortest": 300, "longest": 1999,
         "drafts": 3, "layers": 4, "heads": 8, "width": 128, "page": 64, "layout": "slots"},
        # the logits of one user
        {"name": "logits_one", "op": "logits", "dtype": "f32", "rows": 1, "drafts": 1, "uneven": False, "tree": "causal",
         "vocabulary": 32_000, "seen": 300, "biases": 0, "allowed": False},
        # a large batch with a large vocabulary, biases and a grammar's mask for each row
        {"name": "logits_batch", "op": "logits", "dtype": "bf16", "rows": 256, "drafts": 1, "uneven": False, "tree": "causal",
         "vocabulary": 128_000, "seen": 4000, "biases": 50, "allowed": True},
        # the rows of drafted trees: a token counts where it was seen or lies on the row's own path
        {"name": "logits_tree", "op": "logits", "dtype": "f16", "rows": 8, "drafts": 33, "uneven": True, "tree": "tree",
         "vocabulary": 50_001, "seen": 2000, "biases": 9, "allowed": True},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention"] * 4 + ["logits"] * 2 + ["round", "fork"])
    if op == "logits":
        vocabulary = _spread(rng, 200, 200_000)
        rows = _spread(rng, 1, 128)
        drafts = _spread(rng, 1, max(1, min(64, 30_000_000 // (vocabulary * rows))))
        return {"op": op, "dtype": rng.choice(["f32", "f16", "bf16"]), "rows": rows, "drafts": drafts, "uneven": rng.random() < 0.5,
                "tree": rng.choice(["causal", "tree", "pattern"]), "vocabulary": vocabulary, "seen": _spread(rng, 1, 8000),
                "biases": rng.choice([0, 1, 17, min(300, vocabulary)]), "allowed": rng.random() < 0.5}
    heads = rng.choice([1, 2, 3, 4, 8])
    width = rng.choice([64, 80, 96, 128, 128, 192, 256])
    case = {"op": op, "dtype": rng.choice(["bf16", "f16", "f32"]), "heads": heads, "width": width,
            "page": rng.choice([1, 4, 8, 16, 32, 64, 256]), "layout": rng.choice(["slots", "heads"])}
    if op == "attention":
        rows = _spread(rng, 1, 64)
        longest = _spread(rng, 1, min(60_000, 250_000 // rows))
        shortest = _spread(rng, 1, longest)
        drafts = _spread(rng, 1, max(1, min(512, longest, 16_000_000 // (rows * longest))))
        case.update(rows=rows, shortest=shortest, longest=longest, drafts=drafts, uneven=rng.random() < 0.5,
                    tree=rng.choice(["causal", "tree", "pattern"]), q_heads=heads * rng.choice([1, 2, 4, 5, 8]))
        return case
    longest = _spread(rng, 1, 600)
    case.update(layers=rng.choice([1, 2, 3]), shortest=_spread(rng, 1, longest), longest=longest, drafts=_spread(rng, 1, 40))
    if op == "round":
        case.update(rows=_spread(rng, 1, 32), uneven=rng.random() < 0.5)
    else:
        case.update(parents=rng.choice([1, 2, 3]), rows=_spread(rng, 4, 40))
    return case


# ---- what follows from a case alone ---------------------------------------------------------------------------------------------

def _ragged(lo, hi, count):
    """`count` whole numbers from lo to hi, the first of them hi."""
    return [hi if s == 0 else lo + int((hi - lo) * math.modf(0.6180339887 * s)[0]) for s in range(count)]


def _draft_counts(case):
    n = case["drafts"]
    return _ragged(min(1, n) if case.get("uneven") else n, n, case["rows"])


def _lengths(case):
    """Tokens of each sequence, its drafted ones among them (attention) or not (rounds and forks)."""
    if case["op"] == "fork":
        return _ragged(case["shortest"], case["longest"], case["parents"])
    lengths = _ragged(case["shortest"], case["longest"], case["rows"])
    return [max(a, b) for a, b in zip(lengths, _draft_counts(case))] if case["op"] == "attention" else lengths


def _kept(n):
    """Drafted tokens that are accepted of n."""
    return (n + 2) // 3


def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    if case["op"] == "logits":
        rows, vocabulary = sum(_draft_counts(case)), case["vocabulary"]
        nbytes = 2 * size * rows * vocabulary + 4 * case["seen"] * case["rows"] + 8 * case["biases"] * case["rows"]
        return {"bytes": nbytes + (rows * vocabulary // 8 if case["allowed"] else 0), "flops": 3 * rows * vocabulary}
    token = 2 * case["heads"] * case["width"] * size  # K and V of a token in a layer
    if case["op"] == "attention":
        counts, lengths = _draft_counts(case), _lengths(case)
        nbytes = token * sum(lengths) + 2 * size * case["q_heads"] * case["width"] * sum(counts) + 4 * sum(lengths) // case["page"]
        pairs = sum(n * (t - n) + (n * (n + 1) // 2 if case["tree"] != "pattern" else n * n // 2) for n, t in zip(counts, lengths))
        return {"bytes": nbytes, "flops": 4 * case["q_heads"] * case["width"] * pairs}
    if case["op"] == "round":
        counts = _draft_counts(case)
        moved = sum(counts) + sum(_kept(n) for n in counts)
        return {"bytes": 2 * token * case["layers"] * moved, "flops": 0}
    parents, children = _lengths(case), case["rows"] - case["parents"]
    copied = sum(parents[i % len(parents)] % case["page"] for i in range(children))
    return {"bytes": 2 * token * case["layers"] * (copied + children * case["drafts"]), "flops": 0}


# ---- inputs ---------------------------------------------------------------------------------------------------------------------

def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _offsets(counts):
    first = [0]
    for n in counts:
        first.append(first[-1] + n)
    return first


def _pattern(kind, counts, gen):
    """CSR pattern of what each drafted token sees: its way to the root of a random tree, or about half of all. None: those up to itself."""
    if kind == "causal":
        return None
    pos, crd = [0], []
    for n in counts:
        if kind == "tree":
            # nodes hang from one of the last few before them: some depth, some breadth
            back = torch.randint(1, 5, (n,), generator=gen).tolist()
            seen = []
            for i in range(n):
                parent = i - back[i]
                seen.append((seen[parent] if parent >= 0 else []) + [i])
        else:
            seen = [torch.nonzero(torch.rand(n, generator=gen) < 0.5).flatten().tolist() for _ in range(n)]
        for row in seen:
            crd.extend(row)
            pos.append(len(crd))
    return _ints(pos), _ints(crd if crd else [0])[:len(crd)]


def _cache(case, lengths, rows, room, layers, gen, dev_gen):
    """A cache that holds `lengths` tokens in its first rows, in pages of any order, with `room` pages more that are free."""
    page, heads, width, dtype = case["page"], case["heads"], case["width"], DTYPES[case["dtype"]]
    used = [-(-t // page) for t in lengths]
    pages = sum(used) + room
    most = max(used) + -(-case["drafts"] // page) + 1
    order = torch.randperm(pages, generator=gen).tolist()
    table, refs, at = torch.full((rows, most), -1, dtype=torch.int32), torch.zeros(pages, dtype=torch.int32), 0
    for s, n in enumerate(used):
        table[s, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    refs[torch.tensor(order[:at], dtype=torch.int64)] = 1
    shape = (layers, pages, heads, page, width) if case["layout"] == "heads" else (layers, pages, page, heads, width)
    K, V = (torch.randn(shape, dtype=dtype, device=DEV, generator=dev_gen) for _ in range(2))
    if case["layout"] == "heads":
        K, V = K.transpose(2, 3), V.transpose(2, 3)
    length = _ints(lengths + [0] * (rows - len(lengths)))
    return {"K": K, "V": V, "table": table.to(DEV), "len": length, "refs": refs.to(DEV)}


def prepare(case, seed):
    gen = torch.Generator().manual_seed(seed)
    dev_gen = torch.Generator(device=DEV).manual_seed(seed)
    state = {"case": case}
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "logits":
        counts, vocabulary, rows = _draft_counts(case), case["vocabulary"], case["rows"]
        first = _offsets(counts)
        seen_counts = _ragged(case["seen"] // 2, case["seen"], rows)
        # tokens as texts have them: a few often, most hardly ever
        draw_tokens = lambda n: (torch.rand(n, device=DEV, generator=dev_gen) ** 3 * vocabulary).int().clamp_(max=vocabulary - 1)
        state.update(first=_ints(first), tree=_pattern(case["tree"], counts, gen), drafts=draw_tokens(first[-1]),
                     logits=(3 * torch.randn(first[-1], vocabulary, device=DEV, generator=dev_gen)).to(dtype),
                     seen=(_ints(_offsets(seen_counts)), draw_tokens(sum(seen_counts))),
                     repetition=1 + 0.5 * torch.rand(rows, device=DEV, generator=dev_gen),
                     presence=torch.rand(rows, device=DEV, generator=dev_gen),
                     frequency=0.2 * torch.rand(rows, device=DEV, generator=dev_gen), bias=None, allowed=None)
        if case["biases"]:
            at = torch.stack([torch.randperm(vocabulary, device=DEV, generator=dev_gen)[:case["biases"]] for _ in range(rows)])
            state["bias"] = (_ints([case["biases"] * s for s in range(rows + 1)]), at.sort(1).values.int().flatten(),
                             5 * torch.randn(rows * case["biases"], device=DEV, generator=dev_gen))
        if case["allowed"]:
            words = torch.randint(-2 ** 31, 2 ** 31, (first[-1], (vocabulary + 31) // 32), device=DEV, generator=dev_gen)
            state["allowed"] = words.to(torch.int32)
    elif case["op"] == "attention":
        counts, lengths = _draft_counts(case), _lengths(case)
        state.update(_cache(case, lengths, case["rows"], 3, 1, gen, dev_gen))
        state.update(first=_ints(_offsets(counts)), counts=counts, lengths=lengths, tree=_pattern(case["tree"], counts, gen),
                     q=torch.randn(sum(counts), case["q_heads"], case["width"], dtype=dtype, device=DEV, generator=dev_gen),
                     scale=case["width"] ** -0.5)
    else:
        lengths, rows, layers = _lengths(case), case["rows"], case["layers"]
        if case["op"] == "round":
            counts = _draft_counts(case)
            kept = [sorted(torch.randperm(n, generator=gen)[:_kept(n)].tolist()) for n in counts]
            state.update(keep=(_ints(_offsets([len(r) for r in kept])), _ints([j for r in kept for j in r])),
                         base=_ints(lengths))
        else:
            counts = [0] * case["parents"] + [case["drafts"]] * (rows - case["parents"])
            children = list(range(case["parents"], rows))
            state.update(parents=_ints([i % case["parents"] for i in range(len(children))]), children=_ints(children),
                         base=_ints([-1] * case["parents"] + [0] * len(children)))
        # of what is free, as many pages as can be asked for, and some
        room = sum(-(-n // case["page"]) + 2 for n in counts) + 5
        state.update(_cache(case, lengths, rows, room, layers, gen, dev_gen))
        state.update(first=_ints(_offsets(counts)), add=_ints(counts), refused=_ints([0]))
        k, v = (torch.randn(layers, sum(counts), case["heads"], case["width"], dtype=dtype, device=DEV, generator=dev_gen)
                for _ in range(2))
        state.update(k=list(k), v=list(v))
    if own:
        _prepare_own(state)
    return state


# ---- the framework's operators --------------------------------------------------------------------------------------------------

def _prepare_own(state):
    """The descriptors, workspaces and output buffers that a program keeps."""
    import paper_1804_10112_amd as spt
    case = state["case"]
    csr = lambda a, cols, **how: None if a is None else spt.DeviceCSR(a[0], a[1], cols, *a[2:], **how)
    if case["op"] == "logits":
        state["rules"] = spt.LogitRules(
            first=state["first"], tree=csr(state["tree"], case["drafts"]), drafts=state["drafts"],
            seen=csr(state["seen"], case["vocabulary"]), bias=csr(state["bias"], case["vocabulary"], ordered=True, unique=True),
            repetition=state["repetition"], presence=state["presence"], frequency=state["frequency"], allowed=state["allowed"])
        state["out"] = torch.empty_like(state["logits"])
        return
    cache = spt.DeviceCache(state["K"], state["V"], state["table"], state["len"], state["refs"])
    state["cache"] = cache
    if case["op"] == "attention":
        state["pattern"] = csr(state["tree"], case["drafts"])
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty(state["q"].shape[:2], device=DEV)
        state["ws"] = cache.workspace(spt.SPT_CACHE_ATTENTION, case["q_heads"])
    else:
        state["ws"] = cache.workspace(spt.SPT_CACHE_EXTEND)
        if case["op"] == "round":
            state["kept"] = csr(state["keep"], case["drafts"], ordered=True, unique=True)


def _run_own(state):
    import paper_1804_10112_amd as spt
    op = state["case"]["op"]
    if op == "logits":
        spt.spt_adjust_logits(state["logits"], state["rules"], state["out"])
        return state["out"]
    cache = state["cache"]
    if op == "attention":
        spt.spt_cache_attention(cache, 0, state["first"], state["pattern"], state["q"], state["scale"], state["out"], state["lse"],
                                state["ws"])
        return state["out"], state["lse"]
    spt.spt_cache_free(cache, state["base"])  # what the step before took: rejected drafts, answers that have ended
    if op == "fork":
        spt.spt_cache_fork(cache, state["parents"], state["children"])
    spt.spt_cache_extend(cache, state["add"], state["refused"], state["ws"])
    for layer, (k, v) in enumerate(zip(state["k"], state["v"])):
        spt.spt_cache_write(cache, layer, state["first"], k, v)
    if op == "round":
        spt.spt_cache_compact(cache, state["first"], state["kept"])
    return state["K"], state["V"], state["table"], state["len"], state["refs"], state["refused"]


# ---- the same in elementary operations ------------------------------------------------------------------------------------------

def _rows_of(pos, total):
    """The row of each entry of a CSR pattern."""
    rows = torch.arange(pos.numel() - 1, device=DEV)
    return torch.repeat_interleave(rows, (pos[1:] - pos[:-1]).long(), output_size=total)


def _sight(state, s):
    """What the drafted tokens of sequence s see of each other, as a matrix of truth values."""
    counts = state["counts"]
    a, n = sum(counts[:s]), counts[s]
    if state["tree"] is None:
        i = torch.arange(n, device=DEV)
        return i[None, :] <= i[:, None]
    pos, crd = state["tree"]
    part = pos[a:a + n + 1].long()
    lo, hi = part[0], part[-1]
    at = torch.arange(crd.numel(), device=DEV)
    inside = (at >= lo) & (at < hi)
    row = torch.searchsorted(part, at, right=True) - 1
    seen = torch.zeros(n, n, dtype=torch.bool, device=DEV)
    seen[row[inside], crd[inside].long()] = True
    return seen


def _plain_attention(state):
    case, q = state["case"], state["q"]
    page, heads, group = case["page"], case["heads"], case["q_heads"] // case["heads"]
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], device=DEV)
    a = 0
    for s, (n, length) in enumerate(zip(state["counts"], state["lengths"])):
        t = torch.arange(length, device=DEV)
        page_of, slot = state["table"][s, t // page].long(), t % page
        k = state["K"][0, page_of, slot].float().permute(1, 2, 0).contiguous()                       # head, width, token
        v = state["V"][0, page_of, slot].float().permute(1, 0, 2).contiguous()                       # head, token, width
        rows = q[a:a + n].float().reshape(n, heads, group, -1).permute(1, 2, 0, 3).reshape(heads, group * n, -1).contiguous()
        seen = torch.ones(n, length, dtype=torch.bool, device=DEV)
        seen[:, length - n:] = _sight(state, s)
        seen = seen.repeat(group, 1)
        z = torch.matmul(rows, k) * state["scale"]
        z = torch.where(seen, z, -math.inf)
        top = z.max(-1, keepdim=True).values
        top = torch.where(top == -math.inf, 0.0, top)
        p = torch.exp(z - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
        out[a:a + n] = o.reshape(heads, group, n, -1).permute(2, 0, 1, 3).reshape(n, heads * group, -1).to(q.dtype)
        lse[a:a + n] = (top + torch.log(total)).reshape(heads * group, n).t()
        a += n
    return out, lse


def _plain_logits(state):
    case, logits = state["case"], state["logits"]
    rows, vocabulary = logits.shape
    seen_pos, seen_crd = state["seen"]
    sequence = _rows_of(state["first"], rows)
    counts = torch.zeros(case["rows"] * vocabulary, dtype=torch.int32, device=DEV)
    at = _rows_of(seen_pos, seen_crd.numel()) * vocabulary + seen_crd
    counts.index_add_(0, at, torch.ones_like(seen_crd))
    counts = counts.view(case["rows"], vocabulary)[sequence].flatten()
    start = state["first"][:-1].long()[sequence]
    if state["tree"] is None:
        row = torch.arange(rows, device=DEV)
        depth = row - start + 1
        row = torch.repeat_interleave(row, depth)
        before = torch.cumsum(depth, 0) - depth
        node = torch.arange(row.numel(), device=DEV) - before[row]
    else:
        row, node = _rows_of(state["tree"][0], state["tree"][1].numel()), state["tree"][1].long()
    path = state["drafts"][start[row] + node]
    counts.index_add_(0, row * vocabulary + path, torch.ones_like(path))
    counts = counts.view(rows, vocabulary)
    x = logits.float()
    repetition, presence, frequency = (state[name][sequence][:, None] for name in ("repetition", "presence", "frequency"))
    penalised = torch.where(x > 0, x / repetition, x * repetition) - (presence + frequency * counts.float())
    x = torch.where(counts > 0, penalised, x)
    if state["bias"] is not None:
        pos, crd, vals = state["bias"]
        dense = torch.zeros(case["rows"] * vocabulary, device=DEV)
        dense[_rows_of(pos, crd.numel()) * vocabulary + crd] = vals
        x = x + dense.view(case["rows"], vocabulary)[sequence]
    if state["allowed"] is not None:
        bits = (state["allowed"][:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
        x = torch.where(bits.flatten(1)[:, :vocabulary] == 1, x, -math.inf)
    return x.to(logits.dtype)


def _plain_free(state, new_len):
    """Cuts each row to new_len tokens (a negative number or one beyond its length leaves it) and frees the pages behind."""
    page, table, refs, length = state["case"]["page"], state["table"], state["refs"], state["len"]
    after = torch.where(new_len < 0, length, torch.minimum(new_len, length))
    j = torch.arange(table.shape[1], device=DEV)
    gone = (j >= ((after + page - 1) // page)[:, None]) & (j < ((length + page - 1) // page)[:, None])
    pages = table[gone].long()
    refs.index_add_(0, pages, torch.full_like(pages, -1, dtype=torch.int32))
    table[gone] = -1
    length.copy_(after)


def _plain_fork(state):
    parents, children, page = state["parents"].long(), state["children"].long(), state["case"]["page"]
    table, refs, length = state["table"], state["refs"], state["len"]
    held = (length[parents] + page - 1) // page
    rows = torch.where(torch.arange(table.shape[1], device=DEV) < held[:, None], table[parents], -1)
    shared = rows[rows >= 0].long()
    refs.index_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    table[children] = rows
    length[children] = length[parents]


def _plain_extend(state):
    """Rows take the free pages of the lowest numbers, in the rows' order; a last page that others hold too is copied first."""
    page, table, refs, length, add = state["case"]["page"], state["table"], state["refs"], state["len"], state["add"]
    width = table.shape[1]
    held = (length + page - 1) // page
    last = table.gather(1, (held - 1).clamp(min=0)[:, None].long()).flatten()
    copied = (length % page != 0) & (add > 0) & (refs[last.clamp(min=0).long()] > 1)
    fits = length + add <= width * page
    wanted = torch.where(fits & (add > 0), (length + add + page - 1) // page - held + copied, 0)
    end = torch.cumsum(wanted, 0)
    free = torch.nonzero(refs == 0).flatten()
    served = fits & (add >= 0) & ((wanted == 0) | (end <= free.numel()))
    start = held - copied.int()
    j = torch.arange(width, device=DEV)
    new = served[:, None] & (j >= start[:, None]) & (j < (start + wanted)[:, None])
    rank = (end - wanted - start)[:, None] + j
    taken = free[rank[new].long()]
    copied &= served
    source = last[copied].long()
    target = free[(end - wanted)[copied].long()]
    slots = torch.arange(page, device=DEV) < (length % page)[copied][:, None]
    row, slot = torch.nonzero(slots, as_tuple=True)
    for pool in (state["K"], state["V"]):
        for layer in pool:
            layer[target[row], slot] = layer[source[row], slot]
    table[new] = taken.int()
    refs.index_add_(0, source, torch.full_like(source, -1, dtype=torch.int32))
    refs[taken] = 1
    length.copy_(torch.where(served, length + add, length))
    state["refused"].copy_((~served).sum().int())


def _plain_tokens(state):
    """Page and slot of each drafted token."""
    page, first = state["case"]["page"], state["first"]
    total = state["k"][0].shape[0]
    row = _rows_of(first, total)
    drafted = (first[1:] - first[:-1])[row]
    t = state["len"][row] - drafted + torch.arange(total, device=DEV) - first[row]
    return state["table"][row, (t // page).long()].long(), (t % page).long()


def _plain_compact(state):
    """Of the drafted tokens those of `keep` are drawn together behind the others, and the row is cut to them."""
    page, first = state["case"]["page"], state["first"]
    pos, crd = state["keep"]
    row = _rows_of(pos, crd.numel())
    context = state["len"] - (first[1:] - first[:-1])
    source = context[row] + crd
    target = context[row] + torch.arange(crd.numel(), device=DEV) - pos[row]
    table = state["table"]
    for pool in (state["K"], state["V"]):
        for layer in pool:
            moved = layer[table[row, (source // page).long()].long(), (source % page).long()]
            layer[table[row, (target // page).long()].long(), (target % page).long()] = moved
    _plain_free(state, (context + pos[1:] - pos[:-1]).int())


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "attention":
        return _plain_attention(state)
    if op == "logits":
        return _plain_logits(state)
    _plain_free(state, state["base"])
    if op == "fork":
        _plain_fork(state)
    _plain_extend(state)
    pages, slots = _plain_tokens(state)
    for layer, (k, v) in enumerate(zip(state["k"], state["v"])):
        state["K"][layer][pages, slots] = k
        state["V"][layer][pages, slots] = v
    if op == "round":
        _plain_compact(state)
    return state["K"], state["V"], state["table"], state["len"], state["refs"], state["refused"]


# ---- by definition, in 64 bits --------------------------------------------------------------------------------------------------

def _exact_sight(state, s, a, n):
    if state["tree"] is None:
        return torch.tril(torch.ones(n, n, dtype=torch.bool))
    pos, crd = state["tree"]
    pos, crd = pos[a:a + n + 1].tolist(), crd.tolist()
    seen = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        seen[i, crd[pos[i]:pos[i + 1]]] = True
    return seen


def _exact_attention(state):
    case = state["case"]
    page, group = case["page"], case["q_heads"] // case["heads"]
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    a = 0
    for s, (n, length) in enumerate(zip(state["counts"], state["lengths"])):
        pages = state["table"][s, :-(-length // page)].long()
        seen = torch.cat([torch.ones(n, length - n, dtype=torch.bool), _exact_sight(state, s, a, n)], 1).to(DEV)
        some = seen.any(1)
        for h in range(case["heads"]):
            k, v = (state[x][0][pages][:, :, h].reshape(-1, case["width"])[:length].double() for x in "KV")
            for g in range(h * group, (h + 1) * group):
                z = (state["q"][a:a + n, g].double() @ k.t().contiguous() * state["scale"]).masked_fill(~seen, -math.inf)
                total = torch.logsumexp(z, 1)
                lse[a:a + n, g] = total
                out[a:a + n, g] = torch.where(some[:, None], (z - torch.where(some, total, 0.0)[:, None]).exp() @ v, 0.0)
        a += n
    return out, lse


def _exact_logits(state):
    x = state["logits"].double()
    vocabulary, first = x.shape[1], state["first"].tolist()
    seen_pos, bias_pos = state["seen"][0].tolist(), state["bias"][0].tolist() if state["bias"] else None
    tree = None if state["tree"] is None else [t.tolist() for t in state["tree"]]
    per_row = [state[name].double().tolist() for name in ("repetition", "presence", "frequency")]
    for s in range(len(first) - 1):
        history = torch.bincount(state["seen"][1][seen_pos[s]:seen_pos[s + 1]].long(), minlength=vocabulary)
        rep, pres, freq = (p[s] for p in per_row)
        for r in range(first[s], first[s + 1]):
            nodes = list(range(r - first[s] + 1)) if tree is None else tree[1][tree[0][r]:tree[0][r + 1]]
            tokens = state["drafts"][[first[s] + j for j in nodes]].long()
            c = history + torch.bincount(tokens, minlength=vocabulary)
            some = c > 0
            y = x[r][some]
            x[r][some] = torch.where(y > 0, y / rep, y * rep) - pres - freq * c[some].double()
            if bias_pos:
                part = slice(bias_pos[s], bias_pos[s + 1])
                x[r][state["bias"][1][part].long()] += state["bias"][2][part].double()
            if state["allowed"] is not None:
                v = torch.arange(vocabulary, device=DEV)
                x[r][(state["allowed"][r].long()[v // 32] >> (v % 32)) % 2 == 0] = -math.inf
    return x


def _exact_pages(state):
    """The round or fork, sequence by sequence on the host; keys and values follow the slots that the host says."""
    case, page = state["case"], state["case"]["page"]
    table, length, refs, first = (state[x].tolist() for x in ("table", "len", "refs", "first"))
    K, V = state["K"].double(), state["V"].double()
    held = lambda t: -(-t // page)
    if case["op"] == "fork":
        for parent, child in zip(state["parents"].tolist(), state["children"].tolist()):
            table[child], length[child] = list(table[parent]), length[parent]
            for p in table[child][:held(length[child])]:
                refs[p] += 1
    free = [p for p, n in enumerate(refs) if n == 0]
    shared = [n > 1 for n in refs]
    refused = 0
    for s, add in enumerate(state["add"].tolist()):
        n, used = held(length[s]), length[s] % page
        copy = add > 0 and used > 0 and shared[table[s][n - 1]]
        wanted = held(length[s] + add) - n + copy if add > 0 else 0
        if wanted > len(free) or length[s] + add > len(table[s]) * page:
            refused += 1
            continue
        taken, free = free[:wanted], free[wanted:]
        for p in taken:
            refs[p] = 1
        if copy:
            old = table[s][n - 1]
            K[:, taken[0], :used], V[:, taken[0], :used] = K[:, old, :used].clone(), V[:, old, :used].clone()
            refs[old] -= 1
        table[s][n - copy:n - copy + wanted] = taken
        length[s] += add
    k, v = torch.stack(state["k"]).double(), torch.stack(state["v"]).double()
    for s, n in enumerate(state["add"].tolist()):
        at = [(table[s][t // page], t % page) for t in range(length[s] - n, length[s])]
        for i, (p, o) in enumerate(at):
            K[:, p, o], V[:, p, o] = k[:, first[s] + i], v[:, first[s] + i]
        if case["op"] == "round":
            pos, crd = state["keep"][0].tolist(), state["keep"][1].tolist()
            kept = crd[pos[s]:pos[s + 1]]
            for i, j in enumerate(kept):
                (p, o) = at[i]
                K[:, p, o], V[:, p, o] = k[:, first[s] + j], v[:, first[s] + j]
            length[s] += len(kept) - n
            for j in range(held(length[s]), held(length[s] + n - len(kept))):
                refs[table[s][j]] -= 1
                table[s][j] = -1
    return K, V, torch.tensor(table), torch.tensor(length), torch.tensor(refs), torch.tensor([refused])


def exact(case, seed):
    global own
    mine, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = mine
    if case["op"] == "attention":
        return _exact_attention(state)
    if case["op"] == "logits":
        return _exact_logits(state)
    return _exact_pages(state)
