"""The paged cache's own operations against the plain bookkeeping: room, release, forks, new tokens, the accepted path."""
import pytest
import torch

import paper_2502_13652_b200 as c2t
from plain_forms import Pages

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2502_13652_b200 import build
    build.build()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(B=5, layers=2, n_pages=40, page=16, G=2, D=64, max_pages=12, dtype=torch.bfloat16, heads_first=False, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (layers, n_pages, G, page, D) if heads_first else (layers, n_pages, page, G, D)
    pools = [torch.randn(shape, device="cuda", generator=g).to(dtype) for _ in range(2)]
    if heads_first:
        pools = [t.permute(0, 1, 3, 2, 4) for t in pools]
    cache = c2t.KVCache(*pools, *c2t.KVCache.new_state(B, max_pages, n_pages))
    return cache, Pages(cache.table.cpu(), cache.held.cpu(), cache.refs.cpu(), page)


def same(cache, plain):
    torch.cuda.synchronize()
    assert cache.held.tolist() == plain.held.tolist()
    assert torch.equal(cache.table.cpu(), plain.table)
    assert cache.refs.tolist() == plain.refs.tolist()
    assert cache.status.tolist() == plain.status


@pytest.mark.parametrize("n_pages", [1, 5, 39, 40, 700])
@pytest.mark.parametrize("page", [8, 16, 256])
def test_reserve_and_release(n_pages, page):
    cache, plain = make(n_pages=n_pages, page=page, G=1, layers=1)
    for length in ([1, 0, page, page + 1, 3], [page * 3, -1, page * 12 + 1, page * 7, 0], [page * 12] * 5, [page * 2] * 5):
        cache.c2t_cache_reserve(ints(length))
        plain.reserve(length)
        same(cache, plain)
        keep = [page * 2, 1, 1 << 30, -3, page + 1]
        cache.c2t_cache_release(ints(keep))
        plain.release(keep)
        same(cache, plain)
    cache.c2t_cache_release(ints([0] * 5))
    plain.release([0] * 5)
    same(cache, plain)
    assert not cache.refs.any()


def test_free_pages_are_the_lowest_wherever_they_lie():
    """More pages than one round of the search looks at, holes in every part of them, and more slots than a block has threads."""
    n, B = 16384 * 2 + 777, 1500
    cache, plain = make(B=B, n_pages=n, page=8, G=1, layers=1, max_pages=40)
    g = torch.Generator().manual_seed(1)
    refs = (torch.rand(n, generator=g) < 0.7).to(torch.int32)
    refs[:9000] = 1
    cache.refs.copy_(refs)
    plain.refs = refs.clone()
    length = torch.randint(0, 100, (B,), generator=g).tolist()
    cache.c2t_cache_reserve(ints(length))                # (about 9500 pages of 7400)
    plain.reserve(length)
    same(cache, plain)
    assert 0 < sum(s == c2t.ST_NO_PAGE for s in plain.status) < B


@pytest.mark.parametrize("free", [0, 1, 2, 3, 40])
@pytest.mark.parametrize("dtype,heads_first", [(torch.bfloat16, False), (torch.float16, True)])
def test_fork(free, dtype, heads_first):
    B, page = 9, 16
    cache, plain = make(B=B, n_pages=9 + free, page=page, dtype=dtype, heads_first=heads_first, layers=3)
    start = [40, 64, 0, 0, 0, 0, 0, 17, 0]               # 3 + 4 + 2 pages
    cache.c2t_cache_reserve(ints(start))
    plain.reserve(start)
    k, v = cache.k.clone(), cache.v.clone()
    source = [-1, -1, 0, 1, 0, 8, 1, 0, 99]              # 5 asks for a slot that is forked into, 7 is not empty, 8 has no such source
    length = [0, 0, 37, 64, 5, 1, 33, 5, 1]
    forked = torch.full((B,), 7, dtype=torch.int32, device="cuda")
    cache.c2t_cache_fork(ints(source), ints(length), forked)
    made, copies = plain.fork(source, length)
    same(cache, plain)
    assert forked.tolist() == made
    for old, new, n in copies:
        k[:, new, :n], v[:, new, :n] = k[:, old, :n], v[:, old, :n]
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v)
    cache.c2t_cache_release(ints([0, 64, 0, 48, 0, 0, 0, 17, 0]))
    plain.release([0, 64, 0, 48, 0, 0, 0, 17, 0])
    same(cache, plain)


def test_fork_of_lengths_that_are_not_there():
    cache, plain = make(B=4)
    cache.c2t_cache_reserve(ints([20, 0, 0, 0]))
    plain.reserve([20, 0, 0, 0])
    forked = torch.zeros(4, dtype=torch.int32, device="cuda")
    for source, length in (([-1, 0, 0, 0], [0, 33, -1, 32]), ([-1, 0, 0, 3], [0, 0, 20, 0])):
        cache.c2t_cache_fork(ints(source), ints(length), forked)
        made, _ = plain.fork(source, length)
        same(cache, plain)
        assert forked.tolist() == made


@pytest.mark.parametrize("B,max_new,page,G,D,dtype,heads_first", [
    (1, 1, 16, 1, 64, torch.bfloat16, False), (3, 7, 8, 2, 128, torch.float16, True), (5, 60, 32, 3, 64, torch.bfloat16, False),
    (2, 300, 128, 2, 64, torch.float16, False)])
def test_append(B, max_new, page, G, D, dtype, heads_first):
    cache, _ = make(B=B, page=page, G=G, D=D, dtype=dtype, heads_first=heads_first, n_pages=20 * B + 400 // page, max_pages=10 + 500 // page, seed=4)
    start = [(37 * b) % 50 for b in range(B)]
    count = [max_new - (3 * b) % (max_new + 1) for b in range(B)]
    if B > 2:
        count[1], count[2] = 0, max_new + 9              # none; cut to max_new
    cache.c2t_cache_reserve(ints([s + min(c, max_new) for s, c in zip(start, count)]))
    wide = torch.randn(B, max_new, G, 2 * D, device="cuda").to(dtype)
    k_new, v_new = wide[..., :D], wide[..., D:]          # halves of one projection's output, or arrays of their own
    if B % 2:
        k_new, v_new = k_new.contiguous(), v_new.contiguous()
    k, v = cache.k.clone(), cache.v.clone()
    cache.c2t_cache_append(1, k_new, v_new, ints(start), ints(count))
    torch.cuda.synchronize()
    table = cache.table.cpu()
    for b in range(B):
        for j in range(min(count[b], max_new)):
            p = start[b] + j
            k[1, table[b, p // page], p % page] = k_new[b, j]
            v[1, table[b, p // page], p % page] = v_new[b, j]
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v) and not cache.status.any()


def test_append_without_room():
    """Tokens whose position has no page are left out and reported, those of the other slots are written."""
    cache, _ = make(B=3, page=8)
    cache.c2t_cache_reserve(ints([8, 16, 0]))
    k_new = torch.randn(3, 4, 2, 64, device="cuda").to(torch.bfloat16)
    k = cache.k.clone()
    cache.c2t_cache_append(0, k_new, k_new, ints([6, 6, -2]), ints([4, 4, 2]))
    torch.cuda.synchronize()
    table = cache.table.cpu()
    k[0, table[0, 0], 6:8] = k_new[0, :2]
    k[0, table[1, 0], 6:8], k[0, table[1, 1], :2] = k_new[1, :2], k_new[1, 2:]
    assert torch.equal(cache.k, k)
    assert cache.status.tolist() == [c2t.ST_BAD_PAGE, 0, c2t.ST_BAD_PAGE]


@pytest.mark.parametrize("page,dtype,heads_first", [(8, torch.bfloat16, False), (16, torch.float16, True), (64, torch.bfloat16, False)])
def test_compact(page, dtype, heads_first):
    paths = [[0], [0, 1, 2], [0, 3, 7, 9, 30], list(range(0, 33)), [0] + list(range(2, 34)), [0, 1, 5, 6, 7, 8, 9, 10, 11, 12, 13], [0, 5],
             [0, 2, 2], [0, 3, 1], [0, 400], [1, 2]]      # the last four: not ascending, behind the pages, without the root (allowed)
    B, W = len(paths), 33
    cache, _ = make(B=B, layers=3, page=page, dtype=dtype, heads_first=heads_first, n_pages=B * 100 // page + 60, max_pages=20, seed=8)
    prefix = [5, 0, 17, 8, 15, 16, 1, 4, 4, 4, 9]
    cache.c2t_cache_reserve(ints([p + 40 for p in prefix]))
    path = torch.full((B, W), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p)
    accepted = [len(p) - 1 for p in paths]
    accepted[6] = -1                                     # none accepted by any walk: refused
    k, v = cache.k.clone(), cache.v.clone()
    new_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    cache.c2t_cache_compact(ints(prefix), ints(accepted), path.cuda(), new_len)
    torch.cuda.synchronize()
    table = cache.table.cpu()
    good = [b not in (6, 7, 8, 9) for b in range(B)]
    for b in range(B):
        if good[b]:
            at = [(int(table[b, (prefix[b] + i) // page]), (prefix[b] + i) % page) for i in range(40)]
            for pool in (k, v):
                rows = [pool[:, at[i][0], at[i][1]].clone() for i in paths[b]]
                for d, row in enumerate(rows):
                    pool[:, at[d][0], at[d][1]] = row
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v)
    assert new_len.tolist() == [p + (a + 1 if ok else 0) for p, a, ok in zip(prefix, accepted, good)]
    assert cache.status.tolist() == [0 if ok else c2t.ST_BAD_PAGE for ok in good]


def test_pages_behind_four_gigabytes():
    """Element offsets beyond 32 bits: the last page of a pool of 5 GB."""
    n, page, G, D = 5 * (1 << 30) // (16 * 8 * 128 * 2), 16, 8, 128
    k = torch.zeros(1, n, page, G, D, dtype=torch.bfloat16, device="cuda")
    table, held, refs = c2t.KVCache.new_state(2, 4, n)
    refs[:n - 2] = 1
    cache = c2t.KVCache(k, k.clone(), table, held, refs)
    cache.c2t_cache_reserve(ints([10, 16]))
    assert cache.table[:, 0].tolist() == [n - 2, n - 1]
    new = torch.randn(2, 16, G, D, device="cuda").to(torch.bfloat16)
    cache.c2t_cache_append(0, new, -new, ints([0, 0]), ints([10, 16]))
    cache.c2t_cache_compact(ints([0, 2]), ints([1, 2]), ints([[0, 5, -1], [0, 4, 7]]))
    torch.cuda.synchronize()
    want = new.clone()
    want[0, 1], want[1, 3], want[1, 4] = new[0, 5], new[1, 6], new[1, 9]
    assert torch.equal(cache.k[0, n - 2, :10], want[0, :10]) and torch.equal(cache.v[0, n - 1], -want[1])
    assert not cache.k[0, :n - 2].any() and not cache.status.any()


def test_calls_in_a_captured_graph_on_another_stream():
    """A graph of a step's cache calls from an empty cache, replayed: the same as the calls one by one."""
    cache, plain = make(B=4, page=8, n_pages=64)
    new = torch.randn(4, 6, 2, 64, device="cuda").to(torch.bfloat16)
    prefix, count = ints([3, 9, 0, 14]), ints([6, 6, 6, 6])
    room, accept = prefix + count, ints([2, 0, 3, 1])
    path = ints([[0, 2, 5, -1], [0, -1, -1, -1], [0, 1, 3, 4], [0, 4, -1, -1]])
    new_len = torch.zeros(4, dtype=torch.int32, device="cuda")

    nothing = ints([0] * 4)

    def step():
        cache.c2t_cache_release(nothing)
        cache.c2t_cache_reserve(room)
        for layer in range(2):
            cache.c2t_cache_append(layer, new, new, prefix, count)
        cache.c2t_cache_compact(prefix, accept, path, new_len)
        cache.c2t_cache_release(new_len)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (cache.k, cache.v, cache.table, cache.held, cache.refs, new_len)]
    cache.k.zero_()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for name, t, w in zip(("v", "table", "held", "refs", "new_len"), (cache.v, cache.table, cache.held, cache.refs, new_len), want[1:]):
        assert torch.equal(t, w), name
    held = cache.table[cache.table >= 0].long()
    assert cache.k[0, held].any() and not cache.status.any()


def shared_and_trimmed(trimmed, heads_first=False):
    """Slot 0 of 40 tokens, slot 1 a fork of its first 32 (two pages of 16), one of them back at 20, inside page 1, with room for 24."""
    cache, plain = make(B=3, heads_first=heads_first)
    for length in ([40, 0, 0],):
        cache.c2t_cache_reserve(ints(length))
        plain.reserve(length)
    cache.c2t_cache_fork(ints([-1, 0, -1]), ints([0, 32, 0]), ints([0, 0, 0]))
    plain.fork([-1, 0, -1], [0, 32, 0])
    keep, room = [1 << 20] * 3, [0, 0, 0]
    keep[trimmed], room[trimmed] = 20, 24
    cache.c2t_cache_release(ints(keep))
    plain.release(keep)
    cache.c2t_cache_reserve(ints(room))
    plain.reserve(room)
    same(cache, plain)
    assert cache.refs.tolist().count(2) == 2
    return cache, plain


@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("trimmed", [0, 1])
def test_nothing_is_written_to_a_page_that_another_slot_holds(trimmed, heads_first):
    """A slot that was trimmed into a page which it shares: new tokens and moved nodes are refused, the other slot keeps its tokens bit for bit."""
    cache, plain = shared_and_trimmed(trimmed, heads_first)
    before = [cache.k.clone(), cache.v.clone()]
    new = [torch.randn(3, 8, cache.kv_heads, cache.head_dim, device="cuda").to(cache.k.dtype) for _ in range(2)]
    start, count = [0, 0, 0], [0, 0, 0]
    start[trimmed], count[trimmed] = 20, 4
    cache.c2t_cache_append(1, *new, ints(start), ints(count))
    plain.status[trimmed] |= c2t.ST_BAD_PAGE
    same(cache, plain)
    assert torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])
    cache.status.zero_()
    prefix, accepted, length = [0, 0, 0], [0, 0, 0], ints([7, 7, 7])
    prefix[trimmed], accepted[trimmed] = 18, 1
    if trimmed == 0:                                     # (slot 1's path of one node stays where it is)
        prefix[1] = 20
    cache.c2t_cache_compact(ints(prefix), ints(accepted), ints([[0, 3]] * 3), length)
    torch.cuda.synchronize()
    assert cache.status[trimmed] == c2t.ST_BAD_PAGE and cache.status[1 - trimmed] == 0
    assert length[trimmed] == 18 and length[1 - trimmed] == prefix[1 - trimmed] + 1
    assert torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])


@pytest.mark.parametrize("trimmed", [0, 1])
def test_a_trimmed_slot_goes_on_in_a_fork_of_its_own(trimmed):
    """What the header names as the way on; and alone with its pages, a slot writes to them again."""
    cache, plain = shared_and_trimmed(trimmed)
    other = 1 - trimmed
    source, length, keep = [-1, -1, trimmed], [0, 0, 20], [1 << 20] * 3
    keep[trimmed] = 0
    cache.c2t_cache_fork(ints(source), ints(length), ints([0, 0, 0]))
    _, copies = plain.fork(source, length)
    cache.c2t_cache_release(ints(keep))
    plain.release(keep)
    cache.c2t_cache_reserve(ints([0, 0, 24]))
    plain.reserve([0, 0, 24])
    same(cache, plain)
    assert len(copies) == 1 and copies[0][2] == 4
    before = [cache.k.clone(), cache.v.clone()]
    new = [torch.randn(3, 8, cache.kv_heads, cache.head_dim, device="cuda").to(cache.k.dtype) for _ in range(2)]
    cache.c2t_cache_append(1, *new, ints([0, 0, 20]), ints([0, 0, 4]))
    for pool, tokens in zip(before, new):
        pool[1, int(plain.table[2, 1]), 4:8] = tokens[2, :4]
    same(cache, plain)
    assert torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])
    cache.c2t_cache_release(ints([1 << 20, 1 << 20, 0]))
    start, count = [0, 0, 0], [0, 0, 0]
    start[other], count[other] = 20, 4                   # its pages are its own by now
    cache.c2t_cache_append(0, *new, ints(start), ints(count))
    for pool, tokens in zip(before, new):
        pool[0, int(plain.table[other, 1]), 4:8] = tokens[other, :4]
    torch.cuda.synchronize()
    assert cache.status.tolist() == [0, 0, 0]
    assert torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])
