"""What stands around a draft tree's verification, as measurable cases: the attention of the tree's nodes (or of a prompt's
next chunk, or of a single token) over a paged cache, the cache's own operations (writing new tokens, keeping the accepted
path, forking, growing and trimming sequences), and the penalties, biases and grammar masks on the logits that a level or an
acceptance walk reads.

A case is a dict of plain values; `prepare` makes what a serving loop holds before the call, `run` makes one pass, `work`
states the bytes and operations that it cannot do without, `exact` computes the same in 64 bits from the definition.  With
`own` false the passes are computed by elementary torch operations in 32 bits.
"""
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
DEPTH = 8                      # tree levels behind the root, at most


def _attend(name, **kw):
    """Attention of the new tokens of `batch` sequences, `new` at most, over `prefix` cached ones at most: of a tree, a
    causal chunk, or single tokens (new = 1); window 0 = all keys."""
    c = dict(kind="attend", batch=8, heads=32, kv_heads=8, dim=128, new=60, tree=True, prefix=2048, page=16, window=0,
             sinks=0, dtype="bf16")
    c.update(kw)
    return dict(c, name=name) if name else c


def _cache(name, kind, **kw):
    c = dict(kind=kind, batch=64, kv_heads=8, dim=128, layers=1, prefix=512, new=60, page=16, dtype="bf16")
    c.update(kw)
    return dict(c, name=name) if name else c


def _rules(name, **kw):
    """Logits rows of `batch` sequences: the rows of all nodes of a verified tree (draft=False) or of a level's frontier."""
    c = dict(kind="rules", batch=8, rows=60, vocab=32000, nodes=60, draft=False, history=1000, bias=True, grammar=True,
             dtype="bf16")
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one interactive user, plain decoding early in a conversation: nothing but latency
        _attend("attend_token_b1_kv700_bf16", batch=1, new=1, tree=False, prefix=700),
        # a full batch of plain decoding, ragged lengths: the cache is read once
        _attend("attend_token_b64_kv4096_bf16", batch=64, new=1, tree=False, prefix=4096),
        # one interactive user, a tree of 60 nodes behind a long prompt: few sequences, a long axis
        _attend("attend_tree_b1_kv16000_bf16", batch=1, prefix=16000, heads=64),
        # a handful of users, shared key heads: 240 rows read the same keys
        _attend("attend_tree_b8_kv2048_bf16"),
        # a batch of trees, every head with keys of its own, as the smaller models have
        _attend("attend_tree_b32_kv3000_f16", batch=32, heads=32, kv_heads=32, prefix=3000, dtype="f16"),
        # a prompt that is read in chunks: the second 2048 tokens and more
        _attend("attend_chunk_b2_n2048_kv6000_bf16", batch=2, new=2048, tree=False, prefix=6000),
        # long conversations on a sliding window with four first tokens kept
        _attend("attend_window_b16_kv20000_f16", batch=16, heads=64, dim=64, prefix=20000, page=32, window=1024, sinks=4,
                dtype="f16"),
        # the accepted path of every sequence moves to the front, in all layers at once
        _cache("compact_b64_l32_bf16", "compact", layers=32),
        # the new tokens' keys and values of one layer go to their pages
        _cache("append_b64_n60_bf16", "append"),
        # four continuations of each prompt: children dropped, forked again, and room for a tree of 60 nodes
        _cache("fork_b64_l8_bf16", "fork", layers=8, prefix=2000),
        # one interactive user, a level's frontier, fp32 logits
        _rules("rules_b1_r10_v32000_f32", batch=1, rows=10, nodes=41, draft=True, bias=False, dtype="f32"),
        # a full batch, every node's row under a grammar, the largest vocabulary
        _rules("rules_b64_r60_v128256_bf16", batch=64, vocab=128256),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["token", "tree", "tree", "chunk", "window", "append", "compact", "fork", "rules", "rules"])
    dtype = rng.choice(["bf16", "f16"])
    if kind in ("token", "tree", "chunk", "window"):
        kv_heads = rng.choice([1, 2, 4, 8, 8, 32])
        heads = kv_heads * (1 if kv_heads == 32 else rng.choice([1, 2, 3, 4, 7, 8]))
        c = _attend(None, kv_heads=kv_heads, heads=heads, dim=rng.choice([64, 128]), page=rng.choice([8, 16, 16, 32, 64, 128]),
                    dtype=dtype, prefix=_log_uniform(rng, 20, 24000), batch=_log_uniform(rng, 1, 64))
        c["new"] = 1 if kind == "token" else _log_uniform(rng, 200, 2048) if kind == "chunk" else rng.randint(2, 100)
        c["tree"] = kind in ("tree", "window")
        if kind == "window":
            c["window"], c["sinks"] = _log_uniform(rng, 40, 4000), rng.choice([0, 1, 4, 130])
        while c["batch"] > 1 and (c["batch"] * c["kv_heads"] * c["dim"] * (c["prefix"] + c["new"]) > 3.5e8 or
                                  c["batch"] * c["heads"] * c["new"] * (c["prefix"] + c["new"]) > 5e8):
            c["batch"] = c["batch"] * 2 // 3
        while c["heads"] * c["new"] * (c["prefix"] + c["new"]) > 5e8:
            c["prefix"], c["new"] = c["prefix"] * 2 // 3, max(1, c["new"] * 2 // 3)
        return c
    if kind == "rules":
        draft = rng.random() < 0.5
        c = _rules(None, batch=_log_uniform(rng, 1, 64), rows=rng.randint(1, 16) if draft else rng.randint(2, 80),
                   vocab=rng.choice([32000, 128256, _log_uniform(rng, 4000, 150000)]), draft=draft,
                   history=_log_uniform(rng, 1, 8000), bias=rng.random() < 0.5, grammar=rng.random() < 0.7,
                   dtype=rng.choice(["bf16", "bf16", "f32"]))
        c["nodes"] = rng.randint(c["rows"], 80) if draft else c["rows"]
        while c["batch"] > 1 and c["batch"] * c["rows"] * c["vocab"] > 2.4e8:
            c["batch"] = c["batch"] * 2 // 3
        return c
    c = _cache(None, kind, batch=_log_uniform(rng, 2, 64), kv_heads=rng.choice([1, 2, 8, 32]), dim=rng.choice([64, 128]),
               layers=1 if kind == "append" else rng.choice([1, 4, 16, 32]), prefix=_log_uniform(rng, 20, 3000),
               new=rng.randint(2, 200) if kind == "append" else rng.randint(12, 80), page=rng.choice([8, 16, 32, 64]),
               dtype=dtype)
    while c["batch"] > 4 and c["layers"] * c["batch"] * c["kv_heads"] * c["dim"] * (c["prefix"] + c["new"] + c["page"]) > 1.2e9:
        c["batch"] = c["batch"] * 2 // 3
    while c["layers"] > 1 and c["layers"] * c["batch"] * c["kv_heads"] * c["dim"] * (c["prefix"] + c["new"] + c["page"]) > 1.2e9:
        c["layers"] //= 2
    return c


# ---------------------------------------------------------------- sizes that follow from the case alone

def _prefixes(case):
    """Ragged: between half of the longest and the longest, spread evenly."""
    p = case["prefix"]
    return [p - int(p * 0.5 * (b * 0.6180339887 % 1.0)) for b in range(case["batch"])]


def _news(case):
    """New tokens per sequence: the most for the first, up to a quarter less for the others."""
    n = case["new"]
    return [n - (7 * b) % (n // 4 + 1) for b in range(case["batch"])]


def _accepted(case):
    return [(5 * b + 3) % (DEPTH + 1) for b in range(case["batch"])]


def _pages(tokens, page):
    return -(-tokens // page)


# ---------------------------------------------------------------- inputs

def _tree(g, batch, nodes):
    """Parents [batch, nodes] (root 0 with parent -1, DEPTH levels at most) and levels, in creation order."""
    parent = torch.full((batch, nodes), -1, dtype=torch.int64)
    level = torch.zeros((batch, nodes), dtype=torch.int64)
    pick = torch.rand(batch, nodes, generator=g)
    rows = torch.arange(batch)
    for i in range(1, nodes):
        p = (pick[:, i] * i).long()
        p = torch.where(level[rows, p] >= DEPTH, torch.zeros_like(p), p)
        parent[:, i] = p
        level[:, i] = level[rows, p] + 1
    return parent, level


def _mask_bits(parent):
    """Ancestor-or-self bits [batch, nodes, words] of trees in creation order."""
    batch, nodes = parent.shape
    on = torch.zeros(batch, nodes, nodes, dtype=torch.bool)
    rows = torch.arange(batch)
    for i in range(nodes):
        if i:
            on[:, i] = on[rows, parent[:, i]]
        on[:, i, i] = True
    words = (nodes + 63) // 64
    bits = torch.zeros(batch, nodes, words * 64, dtype=torch.int64)
    bits[:, :, :nodes] = on
    return (bits.view(batch, nodes, words, 64) << torch.arange(64)).sum(3)


def _pool(case, g, tokens, layers=1, spare=0):
    """Pages in shuffled order that hold `tokens` per sequence: k, v [layers, pages, page, kv_heads, dim], table, held, refs."""
    B, page = case["batch"], case["page"]
    held = [_pages(t, page) for t in tokens]
    width = max(held) + _pages(case["new"], page) + 1
    n = sum(held) + spare
    order = torch.randperm(n, generator=g)
    table = torch.full((B, width), -1, dtype=torch.int32)
    refs = torch.zeros(n, dtype=torch.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        refs[order[at:at + held[b]]] = 1
        at += held[b]
    gg = torch.Generator(device="cuda").manual_seed(int(torch.randint(1 << 30, (1,), generator=g)))
    shape = (layers, n, page, case["kv_heads"], case["dim"])
    k = torch.randn(shape, device="cuda", dtype=_TYPES[case["dtype"]], generator=gg)
    v = torch.randn(shape, device="cuda", dtype=_TYPES[case["dtype"]], generator=gg)
    return dict(k=k, v=v, table=table.cuda(), held=torch.tensor(held, dtype=torch.int32).cuda(), refs=refs.cuda()), gg


def _ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def prepare(case, seed):
    g = torch.Generator().manual_seed(seed)
    B = case["batch"]
    if case["kind"] == "rules":
        return _prepare_rules(case, g)
    prefix, new = _prefixes(case), _news(case)
    s = dict(case=case, prefix=_ints(prefix), new=_ints(new))
    dtype, N = _TYPES[case["dtype"]], case["new"]
    if case["kind"] == "attend":
        pool, gg = _pool(case, g, [p + n for p, n in zip(prefix, new)])
        s.update(pool)
        s["q"] = 2 * torch.randn(B, N, case["heads"], case["dim"], device="cuda", dtype=dtype, generator=gg)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(B, N, case["heads"], device="cuda")
        s["bits"] = s["positions"] = None
        if case["tree"]:
            parent, level = _tree(g, B, N)
            s["bits"] = _mask_bits(parent).cuda()
            s["positions"] = (torch.tensor(prefix)[:, None] + level).to(torch.int32).cuda()
    elif case["kind"] == "append":
        pool, gg = _pool(case, g, [p + n for p, n in zip(prefix, new)])
        s.update(pool)
        s["k_new"] = torch.randn(B, N, case["kv_heads"], case["dim"], device="cuda", dtype=dtype, generator=gg)
        s["v_new"] = torch.randn(B, N, case["kv_heads"], case["dim"], device="cuda", dtype=dtype, generator=gg)
    elif case["kind"] == "compact":
        pool, gg = _pool(case, g, [p + n for p, n in zip(prefix, new)], case["layers"])
        s.update(pool)
        path = torch.full((B, DEPTH + 1), -1, dtype=torch.int32)
        for b, a in enumerate(_accepted(case)):
            a = min(a, new[b] - 1)
            path[b, 0] = 0
            path[b, 1:a + 1] = 1 + torch.randperm(new[b] - 1, generator=g)[:a].sort().values
        s["path"], s["length"] = path.cuda(), torch.zeros(B, dtype=torch.int32, device="cuda")
        s["accepted"] = _ints([min(a, n - 1) for a, n in zip(_accepted(case), new)])
    else:                                               # the first fifth of the slots hold prompts, the others continue them
        parents = max(1, B // 5)
        pool, gg = _pool(case, g, prefix[:parents] + [0] * (B - parents), case["layers"],
                         spare=B * (_pages(N, case["page"]) + 2))
        s.update(pool)
        source = [-1] * parents + [b % parents for b in range(parents, B)]
        length = [prefix[b if src < 0 else src] for b, src in enumerate(source)]
        s["source"], s["length"] = _ints(source), _ints(length)
        s["keep"] = _ints(prefix[:parents] + [0] * (B - parents))
        s["room"] = _ints([x + N for x in length])
        s["forked"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    if own:
        import paper_2502_13652_b200 as c2t
        heads = dict(q_heads=case["heads"], max_queries=N) if case["kind"] == "attend" else {}
        s["cache"] = c2t.KVCache(s["k"], s["v"], s["table"], s["held"], s["refs"], **heads)
    return s


def _prepare_rules(case, g):
    B, R, V, N = case["batch"], case["rows"], case["vocab"], case["nodes"]
    pad = -(-V // 8) * 8                                # rows on 16-byte boundaries
    gg = torch.Generator(device="cuda").manual_seed(int(torch.randint(1 << 30, (1,), generator=g)))
    logits = torch.empty(B, R, pad, device="cuda", dtype=_TYPES[case["dtype"]])
    logits.normal_(0.0, 4.0, generator=gg)
    s = dict(case=case, logits=logits[:, :, :V], out=torch.zeros_like(logits)[:, :, :V])
    # words of a text: low ids far more often than high ones
    words = (V * torch.rand(B, case["history"], device="cuda", generator=gg) ** 4).long()
    s["counts"] = torch.zeros(B, V, dtype=torch.int32, device="cuda")
    s["counts"].scatter_add_(1, words, torch.ones_like(words, dtype=torch.int32))
    s["repetition"] = 1.0 + 0.3 * torch.rand(B, device="cuda", generator=gg)
    s["frequency"] = 0.2 * torch.rand(B, device="cuda", generator=gg)
    s["presence"] = 0.5 * torch.rand(B, device="cuda", generator=gg)
    s["bias"] = None
    if case["bias"]:                                    # one table for all sequences, a few hundred tokens in it
        s["bias"] = torch.zeros(V, device="cuda")
        at = torch.randint(V, (300,), device="cuda", generator=gg)
        s["bias"][at] = 5 * torch.randn(300, device="cuda", generator=gg)
    s["allowed"] = None
    if case["grammar"]:                                 # free text for some rows, a tenth of the words for the others
        words = (V + 31) // 32
        on = torch.rand(B, R, words * 32, device="cuda", generator=gg) < 0.1
        on |= (torch.rand(B, R, 1, device="cuda", generator=gg) < 0.3)
        on[:, :, 5] = True
        s["allowed"] = (on.view(B, R, words, 32).long() << torch.arange(32, device="cuda")).sum(3).to(torch.int32)
    parent, _ = _tree(g, B, N)
    s["parent"], s["bits"] = parent.to(torch.int32).cuda(), _mask_bits(parent).cuda()
    s["token"] = (V * torch.rand(B, N, device="cuda", generator=gg) ** 4).to(torch.int32)
    if case["draft"]:                                   # the frontier: the tree's last nodes
        s["row_node"] = torch.arange(N - R, N, dtype=torch.int32, device="cuda").expand(B, R).contiguous()
        n_rows = [R - (3 * b) % (R // 3 + 1) for b in range(B)]
    else:
        s["row_node"] = None
        n_rows = [R - (7 * b) % (R // 4 + 1) for b in range(B)]
    s["n_rows"] = _ints(n_rows)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return {"attend": _run_attend, "append": _run_append, "compact": _run_compact, "fork": _run_fork,
            "rules": _run_rules}[s["case"]["kind"]](s)


def _run_attend(s):
    c = s["case"]
    if own:
        s["cache"].c2t_verify_attention(0, s["q"], s["out"], s["new"], s["prefix"], mask_bits=s["bits"],
                                        position_ids=s["positions"], window=c["window"], sinks=c["sinks"], lse=s["lse"])
        return s["out"], s["lse"]
    B, N, H, G, D = c["batch"], c["new"], c["heads"], c["kv_heads"], c["dim"]
    length = c["prefix"] + N
    width = _pages(length, c["page"])
    pages = s["table"][:, :width].clamp(min=0).long()
    live = (torch.arange(length, device="cuda") < (s["prefix"] + s["new"])[:, None])
    keys = s["k"][0][pages].reshape(B, width * c["page"], G, D)[:, :length].float()
    values = s["v"][0][pages].reshape(B, width * c["page"], G, D)[:, :length].float()
    q = s["q"].float().view(B, N, G, H // G, D)
    score = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(B, G, H // G * N, D), keys.permute(0, 2, 3, 1)) * D ** -0.5
    seen = _seen(s, length) & live[:, None, :]                                             # [B, N, length]
    score = score.view(B, G, H // G, N, length).masked_fill_(~seen[:, None, None], -torch.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top > -torch.inf, top, torch.zeros_like(top))
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    mixed = torch.matmul(weight.view(B, G, H // G * N, length), values.permute(0, 2, 1, 3)).view(B, G, H // G, N, D)
    mixed = torch.where(total > 0, mixed / total, torch.zeros_like(mixed)).permute(0, 3, 1, 2, 4).reshape(B, N, H, D)
    lse = (top + total.log()).permute(0, 3, 1, 2, 4).reshape(B, N, H)
    row = (torch.arange(N, device="cuda") < s["new"][:, None])
    return (torch.where(row[:, :, None, None], mixed.to(s["out"].dtype), s["out"]),
            torch.where(row[:, :, None], lse, s["lse"]))


def _seen(s, length):
    """Which of the sequence's keys each new token may see: [B, N, length]."""
    c = s["case"]
    N = c["new"]
    key = torch.arange(length, device="cuda")
    node = key[None, :] - s["prefix"][:, None]                                              # [B, length]
    inside = node.clamp(0, N - 1)
    if s["bits"] is None:
        position = s["prefix"][:, None] + torch.arange(N, device="cuda")
        on = node[:, None, :] <= torch.arange(N, device="cuda")[:, None]
    else:
        position = s["positions"]
        word = torch.gather(s["bits"], 2, (inside // 64)[:, None, :].expand(-1, N, -1))
        on = (word >> (inside % 64)[:, None, :]) & 1 > 0
    on = torch.where((node < 0)[:, None, :], torch.ones_like(on), on)
    if c["window"]:
        at = torch.where(node < 0, key[None, :].expand_as(node), torch.gather(position, 1, inside))
        on = on & ((position[:, :, None] - at[:, None, :] < c["window"]) | (at < c["sinks"])[:, None, :])
    return on


def _run_append(s):
    if own:
        s["cache"].c2t_cache_append(0, s["k_new"], s["v_new"], s["prefix"], s["new"])
        return s["k"], s["v"]
    c = s["case"]
    j = torch.arange(c["new"], device="cuda").expand(c["batch"], -1)
    j = torch.where(j < s["new"][:, None], j, 0)         # a place behind a sequence's last token is its first once more
    at = s["prefix"][:, None] + j
    place = torch.gather(s["table"], 1, at // c["page"]).long() * c["page"] + at % c["page"]
    tokens = (torch.arange(c["batch"], device="cuda")[:, None] * c["new"] + j).reshape(-1)
    for pool, new in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
        pool[0].view(-1, c["kv_heads"], c["dim"])[place.reshape(-1)] = new.view(-1, c["kv_heads"], c["dim"])[tokens]
    return s["k"], s["v"]


def _move_tokens(s, source, target):
    """Tokens of every layer from the places `source` to `target` (page * page size + offset), all read before one is written."""
    layers, pages, page, G, D = s["k"].shape
    for pool in (s["k"], s["v"]):
        rows = pool.view(layers, pages * page, G, D)
        rows[:, target] = rows[:, source]


def _run_compact(s):
    if own:
        s["cache"].c2t_cache_compact(s["prefix"], s["accepted"], s["path"], s["length"])
        return s["k"], s["v"], s["length"]
    page = s["case"]["page"]
    step = torch.arange(DEPTH + 1, device="cuda")
    keep = step <= s["accepted"][:, None]                # the others move the root's token onto itself
    source = s["prefix"][:, None] + torch.where(keep, s["path"], 0)
    target = s["prefix"][:, None] + torch.where(keep, step, 0)
    source, target = (torch.gather(s["table"], 1, at // page).long() * page + at % page for at in (source, target))
    _move_tokens(s, source.reshape(-1), target.reshape(-1))
    s["length"].copy_(s["prefix"] + s["accepted"] + 1)
    return s["k"], s["v"], s["length"]


def _run_fork(s):
    if own:
        s["cache"].c2t_cache_release(s["keep"])
        s["cache"].c2t_cache_fork(s["source"], s["length"], s["forked"])
        s["cache"].c2t_cache_reserve(s["room"])
        return s["table"], s["held"], s["refs"], s["forked"], s["k"], s["v"]
    c = s["case"]
    page, table, refs = c["page"], s["table"], s["refs"]
    column = torch.arange(table.shape[1], device="cuda")
    # the pages behind `keep` go back
    kept = torch.minimum(s["held"], (s["keep"] + page - 1) // page)
    drop = (column >= kept[:, None]) & (column < s["held"][:, None])
    refs.index_add_(0, torch.where(drop, table, 0).reshape(-1).long(), -drop.reshape(-1).to(torch.int32))
    table.copy_(torch.where(drop, -1, table))
    # whole pages are shared, a started one is copied to a page of its own
    fork = s["source"] >= 0
    src = s["source"].clamp(min=0).long()
    full, rest = s["length"] // page, s["length"] % page
    share = fork[:, None] & (column < full[:, None])
    refs.index_add_(0, torch.where(share, table[src], 0).reshape(-1).long(), share.reshape(-1).to(torch.int32))
    table.copy_(torch.where(share, table[src], table))
    copy = fork & (rest > 0)
    fresh = _take_free(refs, copy.to(torch.int32)[:, None].expand(-1, 1))[:, 0]
    started = torch.gather(table[src], 1, full[:, None].long())[:, 0]
    refs.index_add_(0, torch.where(copy, fresh, 0).long(), copy.to(torch.int32))
    table.copy_(torch.where(copy[:, None] & (column == full[:, None]), fresh[:, None].to(torch.int32), table))
    at = torch.arange(page, device="cuda")
    move = copy[:, None] & (at < rest[:, None])
    still = table[0, 0].long() * page                    # what does not move is the first prompt's first token, onto itself
    source = torch.where(move, started.clamp(min=0).long()[:, None] * page + at, still)
    target = torch.where(move, fresh.long()[:, None] * page + at, still)
    _move_tokens(s, source.reshape(-1), target.reshape(-1))
    held = torch.where(fork, full + copy, kept)
    # room for what comes
    want = torch.maximum(held, (s["room"] + page - 1) // page)
    grow = (column >= held[:, None]) & (column < want[:, None])
    fresh = _take_free(refs, grow.to(torch.int32))
    refs.index_add_(0, torch.where(grow, fresh, 0).reshape(-1).long(), grow.reshape(-1).to(torch.int32))
    table.copy_(torch.where(grow, fresh.to(torch.int32), table))
    s["held"].copy_(want)
    s["forked"].copy_(fork)
    return table, s["held"], refs, s["forked"], s["k"], s["v"]


def _take_free(refs, need):
    """The page for each 1 of need [B, n]: free pages in ascending order, for the ones in row order."""
    free = torch.argsort((refs > 0).to(torch.int32), stable=True)
    turn = need.reshape(-1).cumsum(0).view_as(need) - 1
    return free[turn.clamp(0, refs.numel() - 1)]


def _run_rules(s):
    c = s["case"]
    if own:
        import paper_2502_13652_b200 as c2t
        c2t.c2t_penalize_logits(s["logits"], s["out"], n_rows=s["n_rows"], counts=s["counts"], repetition=s["repetition"],
                                frequency=s["frequency"], presence=s["presence"], bias=s["bias"], allowed=s["allowed"],
                                node_token=s["token"], node_parent=s["parent"], row_node=s["row_node"])
        return s["out"]
    B, R, V, N = c["batch"], c["rows"], c["vocab"], c["nodes"]
    bits = s["bits"] if s["row_node"] is None else torch.gather(
        s["bits"], 1, s["row_node"].long()[:, :, None].expand(-1, -1, s["bits"].shape[2]))
    node = torch.arange(N, device="cuda")
    on = (bits[:, :, node // 64] >> (node % 64)) & 1                                        # [B, R, N]
    count = s["counts"][:, None, :].expand(B, R, V).float()
    count = count.scatter_add(2, s["token"].long()[:, None, :].expand(B, R, N), on.float())
    x = s["logits"].float()
    rep = s["repetition"][:, None, None]
    x = torch.where(count > 0, torch.where(x > 0, x / rep, x * rep), x)
    x = x - s["frequency"][:, None, None] * count
    x = torch.where(count > 0, x - s["presence"][:, None, None], x)
    if s["bias"] is not None:
        x = x + s["bias"]
    if s["allowed"] is not None:
        token = torch.arange(V, device="cuda")
        x = torch.where((s["allowed"][:, :, token // 32] >> (token % 32)) & 1 > 0, x, -torch.inf)
    row = torch.arange(R, device="cuda") < s["n_rows"][:, None]
    return torch.where(row[:, :, None], x.to(s["out"].dtype), s["out"])


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    esz = 4 if case["dtype"] == "f32" else 2
    B = case["batch"]
    if case["kind"] == "rules":
        rows = sum(case["rows"] - ((3 if case["draft"] else 7) * b) % (case["rows"] // (3 if case["draft"] else 4) + 1)
                   for b in range(B))
        V = case["vocab"]
        moved = 2 * rows * V * esz + 4 * B * V + (4 * V if case["bias"] else 0) + (rows * V // 8 if case["grammar"] else 0)
        return {"bytes": moved + 8 * B * case["nodes"], "flops": 6 * rows * V}
    prefix, new = _prefixes(case), _news(case)
    token = 2 * case["kv_heads"] * case["dim"] * esz                                        # key and value of one token
    if case["kind"] == "attend":
        keys = pairs = 0
        for p, n in zip(prefix, new):
            if case["window"]:
                first = min(p, case["sinks"])
                keys += min(p, first + case["window"] - 1) + n
                pairs += n * min(p, first + case["window"]) + n
            else:
                keys += p + n
                pairs += n * p + (n * (n + 1) // 2 if not case["tree"] else n * min(n, DEPTH // 2))
        rows = sum(new) * case["heads"]
        return {"bytes": keys * token + 2 * rows * case["dim"] * esz + 4 * rows, "flops": 4 * case["heads"] * case["dim"] * pairs}
    if case["kind"] == "append":
        return {"bytes": 2 * sum(new) * token, "flops": 0}
    if case["kind"] == "compact":
        return {"bytes": 2 * case["layers"] * sum(min(a, n - 1) for a, n in zip(_accepted(case), new)) * token + 4 * B, "flops": 0}
    parents = max(1, B // 5)
    forks = [prefix[b % parents] for b in range(parents, B)]
    tables = sum(_pages(p, case["page"]) for p in prefix[:parents]) + sum(_pages(p + case["new"], case["page"]) for p in forks)
    return {"bytes": 2 * case["layers"] * token * sum(p % case["page"] for p in forks) + 24 * tables, "flops": 0}


# ---------------------------------------------------------------- the same in 64 bits, from the definition

def exact(case, seed):
    if case["kind"] not in ("attend", "rules"):
        return None                                     # these move values and count pages
    s = prepare(case, seed)
    return _exact_attend(s) if case["kind"] == "attend" else _exact_rules(s)


def _exact_attend(s):
    """Sequence by sequence and key head by key head: softmax over the visible keys, in order of position."""
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    out, lse = s["out"].double(), s["lse"].double()
    for b in range(c["batch"]):
        p, n = int(s["prefix"][b]), int(s["new"][b])
        pages = s["table"][b, :_pages(p + n, c["page"])].long()
        see = torch.ones(n, p + n, dtype=torch.bool, device="cuda")
        where = torch.arange(p + n, device="cuda")
        if s["bits"] is None:
            see[:, p:] = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        else:
            see[:, p:] = torch.stack([(s["bits"][b, :n, j // 64] >> (j % 64)) & 1 for j in range(n)], 1).bool()
            where[p:] = s["positions"][b, :n]
        if c["window"]:
            see &= (where[p:, None] - where[None, :] < c["window"]) | (where < c["sinks"])[None, :]
        for h in range(c["kv_heads"]):
            k = s["k"][0, pages, :, h].reshape(-1, c["dim"])[:p + n].double()
            v = s["v"][0, pages, :, h].reshape(-1, c["dim"])[:p + n].double()
            x = torch.einsum("ngd,kd->gnk", s["q"][b, :n, h * group:(h + 1) * group].double(), k) / c["dim"] ** 0.5
            x = x.masked_fill(~see, -torch.inf)
            out[b, :n, h * group:(h + 1) * group] = torch.einsum("gnk,kd->ngd", torch.softmax(x, -1), v)
            lse[b, :n, h * group:(h + 1) * group] = torch.logsumexp(x, -1).T
    return out, lse


def _exact_rules(s):
    """Row by row: the history's counts and the tokens on the row's own root path."""
    c = s["case"]
    out = s["out"].double()
    parent, token, n_rows = s["parent"].tolist(), s["token"].tolist(), s["n_rows"].tolist()
    for b in range(c["batch"]):
        rep, freq, pres = (s[k][b].double() for k in ("repetition", "frequency", "presence"))
        for r in range(n_rows[b]):
            times = s["counts"][b].clone()
            node = r if s["row_node"] is None else c["nodes"] - c["rows"] + r
            while node >= 0:
                times[token[b][node]] += 1
                node = parent[b][node]
            times = times.double()
            x = s["logits"][b, r].double()
            x = torch.where(times > 0, torch.where(x > 0, x / rep, x * rep) - pres, x) - freq * times
            if s["bias"] is not None:
                x = x + s["bias"].double()
            if s["allowed"] is not None:
                on = (s["allowed"][b, r][:, None] >> torch.arange(32, device="cuda")) & 1
                x = x.masked_fill(on.reshape(-1)[:c["vocab"]] == 0, -torch.inf)
            out[b, r] = x
    return out
