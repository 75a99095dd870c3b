"""Attention of new tokens over the paged cache against the plain 64-bit form: trees, chunks and single tokens."""
import math

import pytest
import torch

import paper_2502_13652_b200 as c2t
from plain_forms import attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2502_13652_b200 import build
    build.build()


def tree(g, B, N, depth=7):
    """Ancestor-or-self bits [B, N, W] and levels [B, N] of random trees."""
    W = (N + 63) // 64
    bits, level = torch.zeros(B, N, W, dtype=torch.int64), torch.zeros(B, N, dtype=torch.int32)
    for b in range(B):
        for i in range(N):
            if i:
                p = int(torch.randint(0, i, (1,), generator=g))
                p = 0 if level[b, p] >= depth else p
                bits[b, i], level[b, i] = bits[b, p], level[b, p] + 1
            bits[b, i, i // 64] |= torch.tensor(1 << (i % 64) if i % 64 < 63 else -2 ** 63, dtype=torch.int64)
    return bits, level


class Case:
    def __init__(self, prefix, n, H=4, G=2, D=128, page=16, dtype=torch.bfloat16, Nq=None, is_tree=True, window=0, sinks=0, layers=1, heads_first=False,
                 seed=0, scale=None, sharp=1.0):
        g = torch.Generator().manual_seed(seed)
        self.g, self.B, self.Nq = g, len(prefix), Nq or max(max(n), 1)
        B, Nq = self.B, self.Nq
        self.window, self.sinks, self.scale, self.layer = window, sinks, scale, layers - 1
        held = [-(-(p + max(0, min(m, Nq))) // page) for p, m in zip(prefix, n)]
        n_pages = sum(held) + 3
        shape = (layers, n_pages, G, page, D) if heads_first else (layers, n_pages, page, G, D)
        k, v = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
        self.k, self.v = (t.permute(0, 1, 3, 2, 4) if heads_first else t for t in (k, v))
        self.q = (sharp * torch.randn(B, Nq, H, D, generator=g)).to(dtype)
        order = torch.randperm(n_pages, generator=g).to(torch.int32)
        self.table = torch.full((B, max(held) + 2), -1, dtype=torch.int32)
        at = 0
        for b in range(B):
            self.table[b, :held[b]] = order[at:at + held[b]]
            at += held[b]
        self.held = torch.tensor(held, dtype=torch.int32)
        self.prefix, self.n = (torch.tensor(x, dtype=torch.int32) for x in (prefix, n))
        self.bits = self.positions = None
        if is_tree:
            self.bits, level = tree(g, B, Nq)
            self.positions = self.prefix[:, None] + level
        self.page, self.G, self.H, self.D, self.dtype = page, G, H, D, dtype

    def on_device(self, heads_first=False):
        k, v = (t.permute(0, 1, 3, 2, 4).contiguous().cuda().permute(0, 1, 3, 2, 4) if heads_first else t.cuda() for t in (self.k, self.v))
        refs = torch.zeros(self.k.shape[1], dtype=torch.int32, device="cuda")
        self.cache = c2t.KVCache(k, v, self.table.cuda(), self.held.cuda(), refs, q_heads=self.H, max_queries=self.Nq)
        wide = torch.randn(self.B, self.Nq, self.H + 1, self.D, device="cuda").to(self.dtype)      # rows among others of a projection
        self.dev_q = wide[:, :, :self.H]
        self.dev_q.copy_(self.q)
        self.out = torch.full((self.B, self.H, self.Nq, self.D), 7.0, dtype=self.dtype, device="cuda").permute(0, 2, 1, 3)
        self.lse = torch.full((self.B, self.Nq, self.H), 7.0, device="cuda")
        self.dev = {k: None if t is None else t.cuda() for k, t in dict(mask_bits=self.bits, position_ids=self.positions).items()}
        self.dev_n, self.dev_prefix = self.n.cuda(), self.prefix.cuda()
        return self

    def call(self, **kw):
        self.cache.c2t_verify_attention(self.layer, self.dev_q, self.out, self.dev_n, self.dev_prefix, window=self.window, sinks=self.sinks,
                                        scale=self.scale, lse=self.lse, **dict(self.dev, **kw))

    def check(self, heads_first=False, status=None):
        self.on_device(heads_first)
        self.call()
        torch.cuda.synchronize()
        return self.compare(status)

    def want(self):
        held = [int(h) * self.page for h in self.held]
        return attend(self.k[self.layer], self.v[self.layer], self.table, self.q, self.n, self.prefix, self.bits, self.positions, self.window, self.sinks,
                      self.scale, held)

    def compare(self, status=None, want=None):
        out, lse, tol, tol_lse = want or self.want()
        got, got_lse = self.out.cpu().double(), self.lse.cpu().double()
        row = torch.arange(self.Nq)[None, :] < self.n[:, None]
        assert bool((got[~row] == 7.0).all()) and bool((got_lse[~row] == 7.0).all())
        assert bool(torch.isfinite(got[row]).all())
        assert torch.equal(torch.isinf(got_lse[row]), torch.isinf(lse[row]))
        off = (got - out).abs()
        assert bool((off <= tol)[row].all()), (float((off / tol.clamp(min=1e-30))[row].max()), torch.nonzero((off > tol) & row[:, :, None, None])[:4].tolist())
        fine = row[:, :, None] & torch.isfinite(lse)
        off = (got_lse - lse).abs()
        assert bool((off <= tol_lse)[fine].all()), float((off / tol_lse)[fine].max())
        assert self.cache.status.tolist() == (status or [0] * self.B)
        return got


TYPES = [torch.bfloat16, torch.float16]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [8, 16, 128, 256])
def test_single_tokens(D, page, dtype):
    Case([0, 1, 7, 8, 126, 127, 128, 129, 300, 255], [1, 1, 1, 1, 1, 1, 1, 0, 1, 1], D=D, page=page, dtype=dtype, is_tree=False, seed=D + page).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N", [2, 17, 60, 64, 65, 130])
def test_trees(D, N, dtype):
    Case([0, 100, 127, 250, 640], [N, N - 1, max(1, N - 7), 0, N], D=D, dtype=dtype, H=4, G=2, seed=N).check()


@pytest.mark.parametrize("H,G", [(1, 1), (3, 3), (8, 1), (7, 1), (6, 2), (40, 8), (300, 1)])
def test_head_layouts(H, G):
    """One key head for all, one for each, groups that do not divide a tile, a group wider than a tile."""
    Case([33, 128], [5, 9], H=H, G=G, D=64, seed=H).check()
    Case([50], [30], H=H, G=G, D=128, dtype=torch.float16, page=32, seed=H).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [[128, 5], [129, 300], [257, 64], [1, 0]])
def test_chunks(n, dtype):
    Case([0, 200], n, is_tree=False, H=2, G=1, dtype=dtype, D=128, seed=n[0]).check()
    Case([130, 3], n, is_tree=False, H=3, G=1, dtype=dtype, D=64, page=64, seed=n[0]).check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (3, 4), (40, 0), (128, 130), (129, 300), (200, 1), (4000, 2), (5, 1 << 30)])
@pytest.mark.parametrize("is_tree", [True, False])
def test_windows(window, sinks, is_tree):
    Case([0, 5, 127, 600, 1000], [20, 33, 7, 12, 40], D=64, is_tree=is_tree, window=window, sinks=sinks, seed=window, H=4, G=2).check()
    Case([900, 261], [150, 290], D=128, is_tree=is_tree, window=window, sinks=sinks, seed=window, H=2, G=1, dtype=torch.float16).check()


def test_a_window_on_single_tokens():
    Case([0, 130, 999, 128, 256], [1] * 5, D=64, is_tree=False, window=128, sinks=4, seed=3).check()


@pytest.mark.parametrize("layers,heads_first", [(1, True), (3, False), (3, True)])
def test_pools_laid_out_otherwise(layers, heads_first):
    Case([70, 128, 0], [9, 60, 33], layers=layers, heads_first=heads_first, seed=2).check(heads_first)


def test_rows_that_see_nothing():
    """No prefix and no bit: zeros and -inf; the rows beside them see what they see."""
    c = Case([0, 0, 5], [40, 3, 20], D=64, seed=1)
    c.bits[0, 5], c.bits[0, 17:30], c.bits[1], c.bits[2, 3] = 0, 0, 0, 0
    got = c.check()
    assert not got[0, 5].any() and not got[1, :3].any() and got[2, 3].any()


def test_bits_behind_the_tree_and_words_that_are_missing():
    """Bits of nodes at or past n_queries name keys that are not there; with fewer words than nodes the last nodes are not seen."""
    c = Case([20, 140], [30, 60], D=64, seed=6)
    c.bits |= -2 ** 62
    c.check()
    c = Case([20, 140], [90, 128], D=64, seed=6)
    c.bits = c.bits[:, :, :1].contiguous()
    c.check()


def test_positions_below_the_prefix_count_as_it():
    c = Case([100, 300], [30, 30], D=64, seed=6, window=33)
    c.positions -= 40
    c.check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("N,D", [(60, 128), (200, 64), (1, 64)])
def test_numbers_that_are_none_where_no_mask_lets_a_row_see(what, N, D, dtype):
    """Behind the last token of a begun page, in pages of nobody, in keys before the window, in a node that only its own subtree sees."""
    c = Case([100, 517, 0], [N, max(1, N - 11), N], D=D, dtype=dtype, is_tree=N > 1, seed=N, window=300, sinks=3)
    seen = torch.zeros(c.k.shape[1] * c.page, dtype=torch.bool)
    bad = []
    for b in range(3):
        keys = int(c.prefix[b]) + int(c.n[b])
        place = c.table[b, torch.arange(keys) // c.page].long() * c.page + torch.arange(keys) % c.page
        seen[place] = True
        if b == 1:                                       # positions 3 .. 517 - 300 - 8 are before every row's window
            seen[place[3:517 - 300 - 8]] = False
        if N > 1:
            bad.append(place[int(c.prefix[b]) + min(9, int(c.n[b]) - 1)])
            c.bits[b, :, 0] &= ~(1 << 9)                 # node 9 is seen by itself alone
            c.bits[b, 9, 0] |= 1 << 9
    for pool in (c.k, c.v):
        flat = pool[0].reshape(-1, c.G, c.D)
        flat[~seen] = what
        if N > 1:
            flat[bad[0], :, ::3] = what                  # and of sequence 0 node 9, in some dimensions
        pool[0] = flat.view_as(pool[0])
    if N > 1:
        c.n[0] = N
        want = c.want()
        c.on_device()
        c.call()
        torch.cuda.synchronize()
        assert not torch.isfinite(c.out[0, 9]).all()     # its own row gets it
        c.out[0, 9] = 0.0
        c.lse[0, 9] = 0.0
        for t in want:
            t[0, 9] = 0.0
        c.compare(want=want)
    else:
        c.check()


def test_large_logits_and_equal_ones():
    """Logits of some hundreds, where one key takes all, and all-equal rows, where all keys have the same weight."""
    c = Case([400, 90], [40, 12], D=128, seed=4, sharp=30.0)
    c.check()
    c = Case([400, 90], [40, 12], D=64, seed=4, dtype=torch.float16)
    c.q.zero_()
    c.check()
    c = Case([1000], [60], D=128, seed=4)                # a maximum that rises from tile to tile, and one that comes last
    c.k[0] = c.q[0, 0, 0].clamp(-1, 1)
    ramp = torch.linspace(-1, 1, 1060)
    for p in range(1060):
        c.k[0, c.table[0, p // 16], p % 16] *= ramp[p]
    c.check()


def test_scale():
    Case([128, 40], [10, 60], scale=0.5, seed=9).check()
    Case([128, 40], [10, 60], scale=1e-3, seed=9, dtype=torch.float16).check()


def test_more_queries_asked_for_than_there_are():
    c = Case([20, 30], [50, 3], Nq=40, D=64, seed=1)
    c.check()


def test_missing_pages_are_not_seen():
    """A slot whose pages end before its tokens, in the tree and in the prefix; and one that holds none at all."""
    c = Case([100, 100, 40, 60], [30, 30, 30, 30], D=64, seed=1)
    c.held[0], c.held[1], c.held[2] = 7, 3, 0
    got = c.check(status=[c2t.ST_BAD_PAGE] * 3 + [0])
    assert not got[2].any()


def test_page_numbers_out_of_range_are_reported():
    c = Case([100, 100, 40], [30, 30, 30], D=64, seed=1)
    want = c.want()
    c.table[0, 2], c.table[1, 4] = c.k.shape[1], -5
    c.on_device()
    c.call()
    torch.cuda.synchronize()
    assert c.cache.status.tolist() == [c2t.ST_BAD_PAGE, c2t.ST_BAD_PAGE, 0]
    assert bool((c.out[2, :30].cpu().double() - want[0][2, :30]).abs().le(want[2][2, :30]).all())


@pytest.mark.parametrize("B,prefix,N", [(1, 9000, 1), (1, 20000, 60), (3, 5000, 150), (40, 300, 3)])
def test_long_caches(B, prefix, N):
    """Keys that are read by many thread blocks, and many short sequences in one."""
    c = Case([prefix - 700 * b if B < 9 else prefix - 7 * b for b in range(B)], [N - b % 2 if N > 1 else 1 for b in range(B)], H=4, G=2, D=128,
             is_tree=N > 1, seed=N)
    c.check()


def test_repeats_bit_for_bit_and_keeps_nothing():
    """Two calls of different lengths through one workspace, in turn."""
    a = Case([3000, 10], [60, 60], H=8, G=2, seed=1).on_device()
    b = Case([40, 2500], [12, 60], H=8, G=2, seed=2, Nq=60).on_device()
    b.cache._workspace = a.cache._workspace
    seen = []
    for _ in range(3):
        a.call()
        b.call()
        torch.cuda.synchronize()
        seen.append([t.clone() for t in (a.out, a.lse, b.out, b.lse)])
    for s in seen[1:]:
        assert all(torch.equal(x, y) for x, y in zip(s, seen[0]))
    a.compare()
    b.compare()


def test_captured_and_replayed_on_another_stream_with_other_lengths():
    """The lengths are the device's: a graph serves whatever they are when it runs."""
    c = Case([1500, 700, 0], [60, 33, 5], H=8, G=2, seed=5).on_device()
    want = c.want()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    c.call()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        c.call()
    for n in ([60, 33, 5], [1, 60, 0], [60, 33, 5]):
        c.n = torch.tensor(n, dtype=torch.int32)
        c.dev_n.copy_(c.n)
        c.held.copy_((c.prefix + c.n + 15) // 16)
        held = torch.minimum(c.held, torch.tensor([-(-1560 // 16), -(-733 // 16), 1], dtype=torch.int32))
        c.held = held
        c.cache.held.copy_(held)
        c.cache.status.zero_()
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        short = [int(p) + m > int(h) * 16 for p, m, h in zip(c.prefix, n, held)]
        c.compare(status=[c2t.ST_BAD_PAGE if s else 0 for s in short], want=want if n == [60, 33, 5] else None)


def test_keys_behind_four_gigabytes():
    """The first sequence's pages are the pool's last: element offsets beyond 32 bits."""
    c = Case([300], [20], G=8, H=8, page=16, seed=3)
    n = 5 * (1 << 30) // (16 * 8 * 128 * 2)
    k = torch.zeros(1, n, 16, 8, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    last = n - c.k.shape[1]
    k[0, last:], v[0, last:] = c.k[0].cuda(), c.v[0].cuda()
    c.on_device()
    c.cache = c2t.KVCache(k, v, (c.table + last).cuda(), c.held.cuda(), torch.zeros(n, dtype=torch.int32, device="cuda"), q_heads=8, max_queries=20)
    c.call()
    torch.cuda.synchronize()
    c.compare()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,n,H,D", [(1, [1, 0, 1], 4, 128), (60, [60, 17, 1], 4, 64), (60, [3, 60, 0], 8, 128), (150, [150, 70, 9], 4, 128), (40, [40, 7, 30], 6, 64)])
def test_what_dead_query_rows_hold_does_not_matter(N, n, H, D, dtype):
    c = Case([300, 40, 700], n, H=H, D=D, Nq=N, dtype=dtype, seed=N).on_device()
    c.dev_q[(torch.arange(N)[None, :] >= c.n[:, None]).cuda()] = math.nan
    c.call()
    torch.cuda.synchronize()
    c.compare()


@pytest.mark.parametrize("over", [0, 1, 2, (0, 1, 2)])
def test_broadcast_queries(over):
    c = Case([500, 90], [60, 33], H=8, G=2, seed=3)
    for d in over if isinstance(over, tuple) else (over,):
        c.q = c.q.narrow(d, 0, 1).expand(*[c.q.shape[i] if i == d else -1 for i in range(4)])
    c.on_device()
    c.dev_q = c.q.cuda()
    for d in over if isinstance(over, tuple) else (over,):
        c.dev_q = c.dev_q.narrow(d, 0, 1).expand_as(c.q)
    assert 0 in c.dev_q.stride()
    c.call()
    torch.cuda.synchronize()
    c.compare()


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_prefixes_that_no_slot_can_have(window, sinks):
    """Below 0 counts as 0; behind all pages the rows see every page that is held, or, with a window, the sinks."""
    c = Case([100, 100, 0], [5, 5, 70], D=64, is_tree=False, window=window, sinks=sinks)
    c.prefix[0] = 2 ** 31 - 1
    c.on_device()
    c.dev_prefix[2] = -7
    c.call()
    torch.cuda.synchronize()
    c.compare(status=[c2t.ST_BAD_PAGE, 0, 0])


@pytest.mark.parametrize("N", [1, 3])
def test_hundreds_of_sequences(N):
    """More than the thread blocks sum up at once, some without a query."""
    c = Case([(b * 37) % 200 for b in range(500)], [0 if b % 11 == 3 else N for b in range(500)], H=2, G=1, D=64, is_tree=N > 1, seed=N)
    c.check()


@pytest.mark.parametrize("N,window", [(5, 0), (70, 300)])
def test_tables_too_wide_for_an_even_deal(N, window):
    """2^30 tokens a slot: the tiles that there could be are more than 32 bits count, and blocks of rows are then not cut."""
    B = 16
    c = Case([9000 if b == 3 else 100 * b for b in range(B)], [N] * B, H=16, G=16, D=64, page=256, window=window, sinks=2, is_tree=window == 0, seed=1)
    c.on_device()
    table = torch.full((B, 1 << 22), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table.cuda()
    c.cache = c2t.KVCache(c.cache.k, c.cache.v, table, c.cache.held, c.cache.refs, q_heads=16, max_queries=N)
    c.call()
    torch.cuda.synchronize()
    c.compare()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [1, 5, 24, 32, 33, 48, 64, 65, 128, 129, 256, 300])
def test_rows_whose_keys_several_thread_blocks_read(rows, D):
    """Every way in which parts of rows lie and are joined, with sequences that have fewer rows than the call allows."""
    Case([4000, 130, 2500, 0], [rows, max(rows // 2, 1), 1, rows], H=2, G=2, D=D, is_tree=rows % 2 == 0, seed=rows).check()


@pytest.mark.parametrize("B,H,G,N,prefix", [(3, 4, 4, 5, 2000), (2, 8, 2, 60, 1000), (9, 16, 16, 1, 700), (37, 4, 4, 2, 300), (38, 4, 4, 2, 300), (5, 24, 8, 9, 4500)])
def test_pieces_and_even_deals(B, H, G, N, prefix):
    """Fewer blocks of rows than thread blocks, as many (148) and more, of unequal lengths."""
    Case([prefix * (b + 1) // B for b in range(B)], [N] * B, H=H, G=G, D=64, is_tree=N > 2, seed=B).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,H", [(1, 2), (3, 6), (60, 2), (140, 4)])
def test_numbers_that_are_none_behind_a_window_in_a_part(N, H, dtype):
    """The key just behind the first row's window lies in a tile that is read, by a thread block that has a part of the rows."""
    c = Case([3000, 5000], [N, N], H=H, G=2, D=64, is_tree=False, window=1000, dtype=dtype, seed=N)
    for b, p in enumerate((2000, 4000)):
        for t in (c.k, c.v):
            t[0, int(c.table[b, p // 16]), p % 16] = math.nan
    c.check()


def test_two_streams_with_a_workspace_each():
    a = Case([3000, 10], [60, 60], H=8, G=2, seed=1).on_device()
    b = Case([40, 2500], [12, 60], H=8, G=2, seed=2).on_device()
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip((a, b), sides):
            with torch.cuda.stream(s):
                c.call()
    torch.cuda.synchronize()
    a.compare()
    b.compare()


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 40, 2 ** 30 + 2 ** 24, 2 ** 30 + 100, 2 ** 30])
@pytest.mark.parametrize("positions", [False, True])
def test_windows_wider_than_any_cache_hide_nothing(window, positions):
    """Nodes behind a row's own among them, which a mask may let it see: rows of 90 nodes, each of which sees all others."""
    c = Case([100, 3, 0], [90, 40, 1], D=64, seed=2, window=window, sinks=1)
    c.bits.fill_(-1)
    if not positions:
        c.positions = None
    c.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N", [1, 140])
@pytest.mark.parametrize("first", [0, 200, 9000])
def test_a_long_flat_tail_behind_one_large_weight_in_f16(D, N, first):
    """16384 keys whose weights are 2^-25.25 of one key's each: less than half of f16's smallest number, 4e-4 of the row together, and all of it where the
    one key's value is 0.  Beside the usual tolerance each weight may be off by 2^-31 of the largest (half of 2^-30).  The same keys for more sequences
    than there are thread blocks, so that few rows are cut into parts, which have maxima of their own."""
    c = Case([16384], [N], D=D, H=1, G=1, page=64, dtype=torch.float16, is_tree=False, scale=1.0)
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.k[..., 0] = -17.5
    c.v.fill_(1.0)
    page, at = int(c.table[0, first // 64]), first % 64
    c.k[0, page, at, :, 0], c.v[0, page, at] = 0.0, 0.0
    out, lse, tol, tol_lse = c.want()
    assert 3e-4 < float(out[0, 0, 0, 0]) < 5e-4
    tol += (16384 + N) * 2.0 ** -31
    c.B = 160
    c.q, c.table, c.held, c.n, c.prefix, out, lse, tol, tol_lse = (torch.cat([t] * c.B) for t in (c.q, c.table, c.held, c.n, c.prefix, out, lse, tol, tol_lse))
    c.on_device()
    c.call()
    torch.cuda.synchronize()
    c.compare(want=(out, lse, tol, tol_lse))


@pytest.mark.parametrize("page", [8, 256])
@pytest.mark.parametrize("window,sinks,up", [(1, 2 ** 31 - 1, 0), (40, 2 ** 31 - 1, 0), (40, 2 ** 31 - 100, 7), (1, 3, 2 ** 31 - 800), (2 ** 31 - 1, 0, 2 ** 31 - 800),
                                             (2 ** 31 - 700, 3, 2 ** 31 - 800), (5, 2 ** 31 - 1, 2 ** 31 - 800), (5, 2 ** 31 - 760, 2 ** 31 - 800)])
def test_windows_sinks_and_positions_near_32_bits(window, sinks, up, page):
    """Positions `up` behind the usual ones; sequences shorter than a page, whose last box reaches to the left of their first key."""
    c = Case([60, 3, 0, 700, 130], [1, 20, 33, 60, 60], D=64, H=4, G=2, page=page, window=window, sinks=sinks, seed=7)
    c.positions = (c.prefix[:, None] + torch.minimum(c.positions - c.prefix[:, None], torch.tensor(9)) + min(up, 2 ** 31 - 1 - 710)).to(torch.int32)
    c.check()
    c.positions = None
    c.check()
