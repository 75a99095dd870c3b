"""The attention's bounded waits: they outlast rows that are done once more, key by key, and where one runs out the slots that it
concerns are reported."""
import math
import os
import subprocess
import sys

import pytest
import torch

import paper_2502_13652_b200 as c2t
from plain_forms import half_step
from test_gpu_attention import Case

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2502_13652_b200 import build
    build.build()


def repeated(c, b, h, times, tokens):
    """Rows of slot b and head h in 64 bits, over keys that are there `times` often: out, lse and the tolerances of plain_forms.attend."""
    N, D, dtype = c.Nq, c.D, c.dtype
    kk, vv = (pool[0].reshape(-1, c.G, c.D)[tokens, h].double() for pool in (c.k, c.v))
    see = torch.ones(N, len(tokens), dtype=torch.bool)
    see[:, -N:] = ((c.bits[b][:, torch.arange(N) // 64] >> (torch.arange(N) % 64)) & 1).bool()
    q, scale, u = c.q[b, :, h].double(), D ** -0.5, half_step(dtype)
    x = (q @ kk.T * scale).masked_fill(~see, -math.inf)
    top = x.amax(1, keepdim=True)
    w = torch.exp(x - top) * times
    total = w.sum(1, keepdim=True)
    w /= total
    out, lse = w @ vv, (top + total.log())[:, 0]
    away = torch.where(see, scale * D * 2.0 ** -23 * (q.abs() @ kk.abs().T) + 2.0 ** -22 * (q @ kk.T * scale).abs(), 0.0).amax(1)
    return out, lse, u * out.abs() + (u + float(times.sum()) * 2.0 ** -23 + 2.0 ** -18 + 2.1 * away[:, None]) * (w @ vv.abs()), away + 2.0 ** -18


@pytest.mark.parametrize("D,dtype", [(64, torch.bfloat16), (128, torch.float16)])
def test_rows_done_once_more_behind_a_long_prefix(D, dtype):
    """A node that only its own row sees holds a NaN: all other rows of two heads are done once more over 350000 keys, in 4 or 5 seconds, longer than any wait
    lasts otherwise.  The heads and the slot whose tiles the same thread blocks take behind those rows are right, and so are the rows themselves."""
    heads, N, page, prefix = torch.cuda.get_device_properties(0).multi_processor_count, 256, 256, 350000
    c = Case([512, 40], [N, N], H=heads, G=heads, D=D, page=page, dtype=dtype, seed=D)
    c.prefix[0] = prefix                                 # the two pages of the prefix over and over
    tail, rest = divmod(prefix, page)
    table = torch.full((2, tail + 2), -1, dtype=torch.int32)
    assert rest + N <= 2 * page
    table[0, :tail] = c.table[0, torch.arange(tail) % 2]
    table[0, tail] = c.table[0, 2]
    table[0, tail + 1] = [p for p in range(c.k.shape[1]) if p not in set(c.table[c.table >= 0].tolist())][0]
    table[1, :2] = c.table[1, :2]
    c.table, c.held = table, torch.tensor([tail + 2, 2], dtype=torch.int32)
    c.bits[:, :, 0] &= ~(1 << 9)
    c.bits[:, 9, 0] |= 1 << 9
    c.positions = None
    bad = [0, heads - 1]                                 # the first thread block's first head, the last one's last
    place = int(table[0, (prefix + 9) // page]), (prefix + 9) % page
    clean = c.v[0, place[0], place[1]].clone()
    c.v[0, place[0], place[1], bad] = math.nan
    c.on_device()
    c.call()
    torch.cuda.synchronize()
    assert c.cache.status.tolist() == [0, 0]
    c.v[0, place[0], place[1]] = clean
    got, got_lse = c.out.cpu().double(), c.lse.cpu().double()
    for b in range(2):
        end = prefix if b == 0 else 40
        at = torch.arange(prefix - rest if b == 0 else 0, end + N)
        tokens, times = table[b, at // page].long() * page + at % page, torch.ones(len(at), dtype=torch.float64)
        if b == 0:
            again = torch.cat([int(table[0, j]) * page + torch.arange(page) for j in range(2)])
            tokens = torch.cat([again, tokens])
            times = torch.cat([torch.full((page,), float((tail + 1) // 2)), torch.full((page,), float(tail // 2)), times.float()]).double()
            assert float(times.sum()) == prefix + N
        for h in range(heads):
            out, lse, tol, tol_lse = repeated(c, b, h, times, tokens)
            row = torch.ones(N, dtype=torch.bool)
            if b == 0 and h in bad:
                row[9] = False
                assert bool(torch.isnan(got[0, 9, h]).all())
            assert bool(((got[b, :, h] - out).abs() <= tol)[row].all()), (b, h)
            assert bool(((got_lse[b, :, h] - lse).abs() <= tol_lse)[row].all()), (b, h)


GIVE_UP = r"""
import ctypes, sys, torch
sys.path.insert(0, {root!r}); sys.path.insert(0, {tests!r})
import paper_2502_13652_b200 as c2t
from test_gpu_attention import Case
assert c2t.LIB_PATH.endswith("libc2t_debug.so")
limit = ctypes.c_int.in_dll(c2t.lib(), "c2t_debug_attention_wait_limit")
usual = limit.value
cases = [Case([3000, 10, 700], [60, 60, 7], H=8, G=2, seed=1),                            # equal pieces, parts
         Case([100 * b for b in range(40)], [17] * 39 + [0], H=8, G=8, D=64, seed=2),     # an even deal
         Case([2000, 300, 5], [150, 1, 90], H=6, G=2, dtype=torch.float16, seed=3),       # queries thread by thread, both halves of the rows
         Case([200 * b for b in range(16)], [70] * 16, H=16, G=16, D=64, page=256, dtype=torch.float16, seed=4)]      # whole blocks (below)
for at, c in enumerate(cases):
    c.on_device()
    if at == 3:
        table = torch.full((16, 1 << 22), -1, dtype=torch.int32, device="cuda")
        table[:, :c.table.shape[1]] = c.table.cuda()
        c.cache = c2t.KVCache(c.cache.k, c.cache.v, table, c.cache.held, c.cache.refs, q_heads=16, max_queries=70)

    def step(n):
        limit.value = n
        c.cache.status.zero_(); c.out.fill_(7.0); c.lse.fill_(7.0)
        c.call()
        torch.cuda.synchronize()
        limit.value = usual
        return c.out.clone(), c.lse.clone(), c.cache.status.tolist()

    out, lse, status = step(usual)
    assert not any(status)
    c.compare()
    given_up = 0
    for n in (0, 1, 2, 3, 5, 9, 17, 40, 100, 1000):
        some_out, some_lse, status = step(n)
        assert set(status) <= {{0, c2t.ST_INTERNAL}}, status
        for b, s in enumerate(status):
            given_up += s != 0
            assert s or (torch.equal(some_out[b], out[b]) and torch.equal(some_lse[b], lse[b])), (at, n, b)
            assert n > 0 or s == (c2t.ST_INTERNAL if int(c.n[b]) else 0), (at, b)
        again_out, again_lse, status = step(usual)      # and the next call on the same workspace is right
        assert not any(status) and torch.equal(again_out, out) and torch.equal(again_lse, lse)
    assert given_up
print("given-up waits ok")
"""


def test_a_wait_that_runs_out_is_reported_for_every_slot_that_it_concerns():
    from paper_2502_13652_b200 import build
    env = dict(os.environ, C2T_LIBRARY=build.build(debug_bounds=True))
    code = GIVE_UP.format(root=ROOT, tests=os.path.join(ROOT, "tests"))
    out = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=900)
    assert out.returncode == 0, out.stdout[-2000:] + out.stderr[-4000:]
    assert "given-up waits ok" in out.stdout
