"""The paged cache, its attention and the rules on logits as a serving loop uses them, around whole decode steps: a prompt read in two chunks,
a slot forked, then steps of draft levels, verification, acceptance, and the accepted path kept."""
import pytest
import torch

import paper_2502_13652_b200 as c2t
from parity_util import make_configs
from plain_forms import attend, penalize

pytestmark = pytest.mark.gpu

B, V, DEPTH, K, F, N = 4, 2000, 4, 4, 4, 13
H, G, D, LAYERS, PAGE = 4, 2, 64, 2, 16


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2502_13652_b200 import build
    build.build()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Loop:
    def __init__(self, dtype):
        self.dtype, self.g = dtype, torch.Generator(device="cuda").manual_seed(3)
        pools = [self.normal(LAYERS, 90, PAGE, G, D) for _ in range(2)]
        self.most = 60
        self.cache = c2t.KVCache(*pools, *c2t.KVCache.new_state(B, 16, 90), q_heads=H, max_queries=self.most)
        self.kept = [[torch.zeros(LAYERS, 0, G, D, dtype=dtype) for _ in range(2)] for _ in range(B)]         # what the cache has to hold
        self.counts = torch.zeros(B, V, dtype=torch.int32, device="cuda")
        self.length = ints([0] * B)

    def normal(self, *shape):
        return torch.randn(*shape, device="cuda", generator=self.g).to(self.dtype)

    def attend_and_check(self, n, bits=None, positions=None):
        """Attention of n new tokens per slot, already in the cache behind `length`, in the last layer, against the plain form."""
        Nq = bits.shape[1] if bits is not None else self.most
        q = self.normal(B, Nq, H, D)
        out = torch.zeros_like(q)
        self.cache.c2t_verify_attention(LAYERS - 1, q, out, n, self.length, mask_bits=bits, position_ids=positions)
        c = self.cache
        cpu = lambda t: None if t is None else t.cpu()
        want, _, tol, _ = attend(c.k[LAYERS - 1].cpu(), c.v[LAYERS - 1].cpu(), c.table.cpu(), q.cpu(), n.cpu(), self.length.cpu(), cpu(bits), cpu(positions))
        row = torch.arange(Nq)[None] < n.cpu()[:, None]
        assert bool(((out.cpu().double() - want).abs() <= tol)[row].all())

    def append(self, n):
        """New tokens' keys and values in every layer; returns them, [layers, B, most, G, D]."""
        new = [self.normal(LAYERS, B, self.most, G, D) for _ in range(2)]
        self.cache.c2t_cache_reserve(self.length + n)
        for layer in range(LAYERS):
            self.cache.c2t_cache_append(layer, new[0][layer], new[1][layer], self.length, n)
        return [t.cpu() for t in new]

    def keep(self, b, new, which):
        self.kept[b] = [torch.cat((old, t[:, b, which]), 1) for old, t in zip(self.kept[b], new)]

    def check_cache(self):
        torch.cuda.synchronize()
        c = self.cache
        assert not c.status.any()
        assert c.held.tolist() == [-(-k[0].shape[1] // PAGE) for k in self.kept]
        assert self.length.tolist() == [k[0].shape[1] for k in self.kept]
        pages = c.table[c.table >= 0].long()
        assert torch.equal(torch.bincount(pages, minlength=c.n_pages).to(torch.int32), c.refs)
        for b in range(B):
            n = self.kept[b][0].shape[1]
            at = c.table[b, torch.arange(n, device="cuda") // PAGE].long(), torch.arange(n, device="cuda") % PAGE
            for pool, want in zip((c.k, c.v), self.kept[b]):
                assert torch.equal(pool[:, at[0], at[1]].cpu(), want), b


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_steps_of_a_serving_loop(dtype):
    s = Loop(dtype)
    for n in ([50, 23, 0, 5], [17, 0, 0, 60]):           # the prompts, in chunks; slot 2 stays empty
        n = ints(n)
        new = s.append(n)
        s.attend_and_check(n)
        for b in range(B):
            s.keep(b, new, slice(0, int(n[b])))
        s.length = s.length + n
        s.check_cache()
    forked = torch.zeros(B, dtype=torch.int32, device="cuda")
    s.cache.c2t_cache_fork(ints([-1, -1, 0, -1]), s.length[0].expand(B).contiguous(), forked)
    assert forked.tolist() == [0, 0, 1, 0]
    s.kept[2] = list(s.kept[0])
    s.length[2] = s.length[0]
    s.check_cache()

    _, cfg = make_configs(B, V, DEPTH, K, F, N, 0.0, torch.bfloat16, classifier="identity")
    ctx = c2t.Context(cfg)
    rules = dict(repetition=1 + torch.rand(B, device="cuda", generator=s.g), frequency=torch.rand(B, device="cuda", generator=s.g),
                 presence=torch.rand(B, device="cuda", generator=s.g), bias=torch.randn(V, device="cuda", generator=s.g))
    cpu_rules = {k: v.cpu() for k, v in rules.items()}
    root = torch.randint(0, V, (B,), dtype=torch.int32, device="cuda", generator=s.g)
    accepted = []
    for step in range(4):
        ctx.c2t_begin_step(root, s.length)
        for level in range(DEPTH):
            logits = torch.randn(B, F, V, device="cuda", generator=s.g).to(torch.bfloat16)
            out = torch.zeros_like(logits)
            view = ctx.c2t_get_view()
            tree = dict(n_rows=view["frontier_n"], counts=s.counts, node_token=view["tree_token"], node_parent=view["tree_parent"],
                        row_node=view["frontier_node"])
            c2t.c2t_penalize_logits(logits, out, **rules, **tree)
            want, _ = penalize(logits.cpu(), **cpu_rules, **{k: t.cpu() for k, t in tree.items()})
            live = ~want.isnan()
            assert bool(live.any()) and bool(((out.cpu().double() - want).abs() <= 2.0 ** -7 * (1 + want.abs()))[live].all())
            ctx.c2t_expand_level(level, out)
            ctx.c2t_prune(level)
        ctx.c2t_prune(c2t.FINAL)
        ctx.c2t_build_verify()
        ver, nodes = ctx.verify, ctx.verify["n_nodes"]
        new = s.append(nodes)
        s.attend_and_check(nodes, ver["mask_bits"], ver["position_ids"])

        target = torch.randn(B, ctx.Nw, V, device="cuda", generator=s.g).to(torch.bfloat16)
        for b in range(B):                               # a path of another length for each sequence
            row = [int(x) for x in ver["retrieve"][b, (step + b) % int(ver["n_leaves"][b])] if x >= 0][:1 + (b + step) % (DEPTH + 1)]
            for here, nxt in zip(row, row[1:]):
                target[b, here, int(ver["tokens"][b, nxt])] = 90.0
        ruled = target.clone()
        tree = dict(n_rows=nodes, counts=s.counts, node_token=ver["tokens"], node_parent=ver["parents"])
        c2t.c2t_penalize_logits(ruled, ruled, **rules, **tree)                    # in place
        ctx.c2t_accept(ruled)
        new_len = torch.zeros(B, dtype=torch.int32, device="cuda")
        before = s.counts.clone()
        s.cache.c2t_cache_compact(s.length, ctx.accepted["accept_len"], ctx.accepted["path"], new_len)
        c2t.c2t_count_tokens(s.counts, ver["tokens"], ctx.accepted["accept_len"], index=ctx.accepted["path"], plus_one=True)
        s.cache.c2t_cache_release(new_len)
        torch.cuda.synchronize()
        want, _ = penalize(target.cpu(), **cpu_rules, **{k: t.cpu() for k, t in dict(tree, counts=before).items()})
        assert bool(((ruled.cpu().double() - want).abs() <= 2.0 ** -7 * (1 + want.abs()))[~want.isnan()].all())
        for b in range(B):
            path, here = [0], 0
            while True:                                  # the greedy walk over the rows as they were ruled
                token = int(ruled[b, here].float().argmax())
                child = [j for j in range(int(nodes[b])) if int(ver["parents"][b, j]) == here and int(ver["tokens"][b, j]) == token]
                if not child:
                    break
                here = child[0]
                path.append(here)
            assert [int(x) for x in ctx.accepted["path"][b] if x >= 0] == path
            accepted.append(len(path) - 1)
            s.keep(b, new, path)
            for j in path:
                before[b, int(ver["tokens"][b, j])] += 1
        assert torch.equal(s.counts, before)
        s.length, root = new_len, ctx.accepted["next_token"].clone()
        s.check_cache()
    assert max(accepted) >= 2 and min(accepted) < max(accepted)
    status, _ = ctx.c2t_status()
    assert status == 0
    ctx.close()
