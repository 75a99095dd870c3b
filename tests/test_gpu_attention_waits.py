"""The attention's bounded waits: where one runs out the slots that it concerns are reported."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2502_13652_b200 import build
    build.build()


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
