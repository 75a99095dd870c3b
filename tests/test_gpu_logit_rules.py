"""Penalties, biases and grammar masks on logits rows, and the history's counts, against the plain 64-bit form."""
import math

import pytest
import torch

import paper_2502_13652_b200 as c2t
from plain_forms import half_step, penalize

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2502_13652_b200 import build
    build.build()


def inputs(B, R, V, N, dtype, seed, bias="one", allowed="rows", draft=False):
    g = torch.Generator().manual_seed(seed)
    pad = -(-V // 8) * 8 + 8
    x = 4 * torch.randn(B, R, pad, generator=g)
    x[torch.rand(B, R, pad, generator=g) < 0.02] = -math.inf
    a = dict(counts=torch.randint(0, 6, (B, V), generator=g).clamp(max=3).sub(2).clamp(min=0).to(torch.int32),
             repetition=1 + torch.rand(B, generator=g), frequency=torch.randn(B, generator=g), presence=torch.rand(B, generator=g),
             n_rows=torch.tensor([(R - b) % (R + 1) for b in range(B)], dtype=torch.int32))
    a["bias"] = {"one": torch.randn(V, generator=g), "each": torch.randn(B, V, generator=g), None: None}[bias]
    words = (V + 31) // 32
    if allowed:
        bits = torch.randint(-2 ** 31, 2 ** 31, (B, R, words + 1), generator=g).to(torch.int32)[:, :, :words]
        bits[0, 0] = 0                                   # nothing allowed
        bits[-1, -1] = -1
        a["allowed"] = bits if allowed == "rows" else bits[:, 0]
    a["node_token"] = torch.randint(0, V, (B, N), generator=g).to(torch.int32)
    a["node_token"][:, :min(N, 4)] = V - 1               # the same token several times on a path, at the row's end
    a["node_parent"] = torch.stack([torch.cat((torch.tensor([-1]), (torch.rand(N - 1, generator=g) * torch.arange(1, N)).long())) for _ in range(B)]).to(torch.int32)
    a["row_node"] = torch.randint(-1, N + 1, (B, R), generator=g).to(torch.int32) if draft else None
    return x.to(dtype)[:, :, :V], a


def check(x, a, in_place=False):
    """Four roundings to 32 bits of terms no larger than their sum of magnitudes, then one to the output's type."""
    want, touched = penalize(x, **a)
    want = torch.where(torch.isinf(want.to(x.dtype)), want.to(x.dtype).double(), want)         # (what the type cannot hold)
    dev = {k: None if t is None else t.cuda() for k, t in a.items()}
    wide = torch.full((x.shape[0], x.shape[1], x.stride(1)), 7.0, dtype=x.dtype, device="cuda")
    src = wide.clone()[:, :, :x.shape[2]]
    src.copy_(x)
    out = src if in_place else wide[:, :, :x.shape[2]]
    before = out.clone()
    c2t.c2t_penalize_logits(src, out, **dev)
    torch.cuda.synchronize()
    got, before = out.cpu(), before.cpu()
    still = want.isnan() & ~x.double().isnan()
    assert torch.equal(got[still], before[still])
    mine = ~still
    assert torch.equal(got[mine].isnan(), want[mine].isnan())
    ok = mine & ~want.isnan()
    assert torch.equal(torch.isinf(got[ok]), torch.isinf(want[ok])) and torch.equal(got[ok].sign()[torch.isinf(got[ok])], want[ok].sign()[torch.isinf(want[ok])].to(got.dtype))
    ok &= torch.isfinite(want)
    full = lambda t: torch.zeros(x.shape, dtype=torch.float64) if t is None else t.double()
    c = full(None) + (0 if a.get("counts") is None else a["counts"].double()[:, None]) + 33
    size = x.double().abs().nan_to_num(0, 0, 0) * (1 if a.get("repetition") is None else a["repetition"].double()[:, None, None])
    if a.get("frequency") is not None:
        size = size + a["frequency"].double().abs()[:, None, None] * c
    if a.get("presence") is not None:
        size = size + a["presence"].double()[:, None, None]
    if a.get("bias") is not None:
        size = size + (a["bias"] if a["bias"].dim() == 1 else a["bias"][:, None]).double().abs()
    tol = half_step(x.dtype) * want.abs() + 4 * 2.0 ** -24 * size * (1 + half_step(x.dtype))
    off = (got.double() - want).abs()
    assert bool((off <= tol)[ok].all()), float((off - tol)[ok].max())
    return got, touched


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,R,V,N", [(1, 1, 1, 1), (2, 3, 7, 5), (3, 5, 2048, 9), (2, 33, 2049, 33), (1, 40, 5003, 70), (2, 9, 1023, 12)])
@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_rules(B, R, V, N, dtype, draft, in_place):
    x, a = inputs(B, R, V, N, dtype, seed=V + N, bias="one" if draft else "each", allowed="rows" if in_place else "one", draft=draft)
    check(x, a, in_place)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("only", ["counts", "bias", "allowed", "tree", "n_rows", "nothing", "no_tree", "no_counts"])
def test_each_rule_alone(only, dtype):
    x, a = inputs(3, 6, 777, 8, dtype, seed=5)
    keys = {"counts": ("counts", "repetition", "frequency", "presence"), "tree": ("node_token", "node_parent", "repetition"), "nothing": (),
            "no_tree": tuple(k for k in a if not k.startswith(("node", "row"))), "no_counts": tuple(k for k in a if k != "counts")}.get(only, (only,))
    got, _ = check(x, {k: a[k] for k in keys})
    if only == "nothing":
        assert torch.equal(got, x)


def test_logits_that_are_no_numbers():
    """NaN and infinities pass where a token is allowed; a token that is not allowed is -inf whatever its logit."""
    x, a = inputs(1, 4, 300, 4, torch.float32, seed=3)
    x[:, :, ::7], x[:, :, 1::7], x[:, :, 2::7] = math.nan, math.inf, -math.inf
    x[:, :, 3::7] = torch.finfo(torch.float32).min
    a["frequency"] = a["frequency"].abs()
    got, _ = check(x, a)
    off = ((a["allowed"].long()[..., torch.arange(300) // 32] >> (torch.arange(300) % 32)) & 1) == 0
    live = torch.arange(4)[None, :, None] < a["n_rows"][:, None, None]
    assert bool((got[off & live] == -math.inf).all())


def test_paths_of_every_length_and_broken_ones():
    """A chain longer than a path may be, a cycle, a parent out of range: followed over 33 nodes at most."""
    V, N = 64, 50
    x = torch.randn(1, N, V)
    chain = torch.arange(-1, N - 1, dtype=torch.int32)[None].clone()
    token = (torch.arange(N, dtype=torch.int32) % 5)[None].clone()
    for parent in (chain, torch.full((1, N), 3, dtype=torch.int32), torch.full((1, N), N, dtype=torch.int32)):
        check(x, dict(node_token=token, node_parent=parent, frequency=torch.ones(1), presence=torch.zeros(1)))


def test_many_nodes():
    """Node arrays that need more shared memory than a kernel has by default."""
    x, a = inputs(2, 5, 400, 8192, torch.bfloat16, seed=11, draft=True)
    check(x, a)


def test_node_arrays_that_fit_alone_but_not_beside_a_blocks_own():
    x, a = inputs(2, 5, 400, 2900, torch.float32, seed=12, draft=True)
    check(x, a)


def test_counts():
    B, V, N = 3, 50, 9
    tokens = torch.randint(0, V, (B, N), dtype=torch.int32)
    tokens[0, 1], tokens[0, 2] = V, -1                  # skipped
    tokens[1] = 7
    counts = torch.zeros(B, V + 6, dtype=torch.int32, device="cuda")[:, :V]
    index = torch.tensor([[0, 1, 2, 3], [0, 2, 4, -1], [0, 9, 8, 8]], dtype=torch.int32)
    for n, idx, plus, delta in ((torch.tensor([9, 20, 0]), None, False, 1), (torch.tensor([3, 2, 3]), index, True, 1), (torch.tensor([-1, 1, -5]), index, True, -1)):
        before = counts.cpu().clone()
        c2t.c2t_count_tokens(counts, tokens.cuda(), n.to(torch.int32).cuda(), None if idx is None else idx.cuda(), plus_one=plus, delta=delta)
        for b in range(B):
            for k in range(min(int(n[b]) + plus, N if idx is None else 4)):
                at = k if idx is None else int(idx[b, k])
                if 0 <= at < N and 0 <= tokens[b, at] < V:
                    before[b, tokens[b, at]] += delta
        assert torch.equal(counts.cpu(), before)
