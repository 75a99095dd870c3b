"""What the calls on a paged cache and on logits rows refuse, before anything runs.  No GPU."""
import ctypes as C

import pytest

import paper_2502_13652_b200 as c2t
from paper_2502_13652_b200 import build
from paper_2502_13652_b200.kv_cache import _calls, c2t_attention, c2t_cache, c2t_logit_rules

A = 1 << 20                                             # an address that nobody follows


@pytest.fixture(scope="module")
def L():
    build.build()
    return _calls()


def cache(**kw):
    f = dict(dtype=c2t.BF16, batch=4, layers=2, kv_heads=2, head_dim=128, page_size=16, n_pages=64, max_pages=8, k_dev=A, v_dev=A,
             layer_stride=64 * 16 * 256, page_stride=16 * 256, token_stride=256, head_stride=128, table_dev=A, held_dev=A, refs_dev=A,
             status_dev=A)
    f.update(kw)
    return c2t_cache(*[f[n] for n, _ in c2t_cache._fields_])


BAD_CACHES = [(dict(k_dev=None), c2t.EINVAL), (dict(v_dev=None), c2t.EINVAL), (dict(table_dev=None), c2t.EINVAL), (dict(held_dev=None), c2t.EINVAL),
              (dict(refs_dev=None), c2t.EINVAL), (dict(dtype=c2t.F32), c2t.EINVAL), (dict(dtype=9), c2t.EINVAL), (dict(batch=0), c2t.EINVAL),
              (dict(layers=0), c2t.EINVAL), (dict(kv_heads=0), c2t.EINVAL), (dict(n_pages=0), c2t.EINVAL), (dict(max_pages=0), c2t.EINVAL),
              (dict(page_size=0), c2t.EINVAL), (dict(page_size=4), c2t.ERANGE), (dict(page_size=24), c2t.ERANGE), (dict(page_size=512), c2t.ERANGE),
              (dict(head_dim=96), c2t.ERANGE), (dict(batch=4097), c2t.ERANGE), (dict(max_pages=1 << 27), c2t.ERANGE),
              (dict(max_pages=1 << 25, page_size=16, batch=4096), c2t.ERANGE), (dict(token_stride=64), c2t.EINVAL), (dict(head_stride=-128), c2t.EINVAL),
              (dict(layer_stride=-8), c2t.EINVAL), (dict(k_dev=A + 8), c2t.EALIGN), (dict(v_dev=A + 2), c2t.EALIGN), (dict(page_stride=4100), c2t.EALIGN),
              (dict(token_stride=260), c2t.EALIGN), (dict(head_stride=132), c2t.EALIGN), (dict(layer_stride=12), c2t.EALIGN)]


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_caches_that_every_call_refuses(L, bad, code):
    c = C.byref(cache(**bad))
    assert L.c2t_cache_reserve(c, A, None) == code
    assert L.c2t_cache_release(c, A, None) == code
    assert L.c2t_cache_fork(c, A, 2 * A, 3 * A, None) == code
    assert L.c2t_cache_append(c, 0, A, A, 4, 1024, 256, 128, A, A, None) == code
    assert L.c2t_cache_compact(c, A, A, A, 7, 2 * A, None) == code
    assert L.c2t_verify_attention(c, C.byref(attention()), A, 1 << 40, None) == code
    assert L.c2t_verify_attention_workspace_bytes(c, 8, 60) == 0


def test_missing_arrays_and_arguments_out_of_range(L):
    c = C.byref(cache())
    assert L.c2t_cache_reserve(None, A, None) == c2t.EINVAL
    assert L.c2t_cache_reserve(c, None, None) == c2t.EINVAL
    assert L.c2t_cache_release(c, None, None) == c2t.EINVAL
    for args in ((None, A, 2 * A), (A, None, 2 * A), (A, 2 * A, None), (A, 2 * A, A), (A, 2 * A, 2 * A)):
        assert L.c2t_cache_fork(c, *args, None) == c2t.EINVAL
    for layer, k, v, most, seq, tok, head, start, count, code in (
            (2, A, A, 4, 1024, 256, 128, A, A, c2t.EINVAL), (-1, A, A, 4, 1024, 256, 128, A, A, c2t.EINVAL), (0, None, A, 4, 1024, 256, 128, A, A, c2t.EINVAL),
            (0, A, None, 4, 1024, 256, 128, A, A, c2t.EINVAL), (0, A, A, 0, 1024, 256, 128, A, A, c2t.EINVAL), (0, A, A, 4, -8, 256, 128, A, A, c2t.EINVAL),
            (0, A, A, 4, 1024, 256, 128, None, A, c2t.EINVAL), (0, A, A, 4, 1024, 256, 128, A, None, c2t.EINVAL), (0, A + 4, A, 4, 1024, 256, 128, A, A, c2t.EALIGN),
            (0, A, A, 4, 1024, 256, 129, A, A, c2t.EALIGN)):
        assert L.c2t_cache_append(c, layer, k, v, most, seq, tok, head, start, count, None) == code
    for prefix, acc, path, width, new, code in ((None, A, A, 7, None, c2t.EINVAL), (A, None, A, 7, None, c2t.EINVAL), (A, A, None, 7, None, c2t.EINVAL),
                                                (A, A, A, 0, None, c2t.EINVAL), (A, A, A, 34, None, c2t.ERANGE), (A, 2 * A, 3 * A, 7, A, c2t.EINVAL),
                                                (A, 2 * A, 3 * A, 7, 2 * A, c2t.EINVAL)):
        assert L.c2t_cache_compact(c, prefix, acc, path, width, new, None) == code


def attention(**kw):
    f = dict(layer=1, q_heads=8, max_queries=60, q_dev=A, out_dev=A, q_seq_stride=60 * 1024, q_token_stride=1024, q_head_stride=128,
             out_seq_stride=60 * 1024, out_token_stride=1024, out_head_stride=128, lse_dev=None, n_queries_dev=A, prefix_len_dev=A, mask_bits_dev=A,
             mask_words=1, position_ids_dev=None, window=0, sinks=0, scale=0.1)
    f.update(kw)
    return c2t_attention(*[f[n] for n, _ in c2t_attention._fields_])


@pytest.mark.parametrize("bad,code", [
    (dict(layer=2), c2t.EINVAL), (dict(layer=-1), c2t.EINVAL), (dict(q_heads=0), c2t.EINVAL), (dict(q_heads=3), c2t.EINVAL), (dict(max_queries=0), c2t.EINVAL),
    (dict(q_dev=None), c2t.EINVAL), (dict(out_dev=None), c2t.EINVAL), (dict(n_queries_dev=None), c2t.EINVAL), (dict(prefix_len_dev=None), c2t.EINVAL),
    (dict(mask_words=0), c2t.EINVAL), (dict(window=-1), c2t.EINVAL), (dict(sinks=-1), c2t.EINVAL), (dict(scale=0.0), c2t.EINVAL),
    (dict(scale=-1.0), c2t.EINVAL), (dict(scale=float("nan")), c2t.EINVAL), (dict(scale=float("inf")), c2t.EINVAL), (dict(q_head_stride=-128), c2t.EINVAL),
    (dict(q_dev=A + 8), c2t.EALIGN), (dict(out_dev=A + 8), c2t.EALIGN), (dict(q_token_stride=1028), c2t.EALIGN), (dict(out_seq_stride=4), c2t.EALIGN)])
def test_attention_that_is_refused(L, bad, code):
    assert L.c2t_verify_attention(C.byref(cache()), C.byref(attention(**bad)), A, 1 << 40, None) == code


def test_attention_workspace(L):
    c = C.byref(cache())
    need = L.c2t_verify_attention_workspace_bytes(c, 8, 60)
    assert need > 0
    a = C.byref(attention())
    assert L.c2t_verify_attention(c, a, None, need, None) == c2t.EINVAL
    assert L.c2t_verify_attention(c, a, A + 16, need, None) == c2t.EALIGN
    assert L.c2t_verify_attention(c, a, A, need - 1, None) == c2t.ERANGE
    assert L.c2t_verify_attention(c, None, A, need, None) == c2t.EINVAL
    for heads, queries in ((0, 60), (3, 60), (8, 0)):
        assert L.c2t_verify_attention_workspace_bytes(c, heads, queries) == 0


def rules(**kw):
    f = dict(dtype=c2t.BF16, batch=2, rows=6, vocab=1000, in_dev=A, out_dev=A, in_seq_stride=6000, in_row_stride=1000, out_seq_stride=6000, out_row_stride=1000,
             n_rows_dev=None, counts_dev=A, counts_stride=1000, repetition_dev=None, frequency_dev=None, presence_dev=None, bias_dev=A, bias_stride=0,
             allowed_dev=A, allowed_seq_stride=192, allowed_row_stride=32, nodes=6, node_token_dev=A, node_parent_dev=A, row_node_dev=None)
    f.update(kw)
    return c2t_logit_rules(*[f[n] for n, _ in c2t_logit_rules._fields_])


@pytest.mark.parametrize("bad,code", [
    (dict(in_dev=None), c2t.EINVAL), (dict(out_dev=None), c2t.EINVAL), (dict(dtype=c2t.F16), c2t.EINVAL), (dict(batch=0), c2t.EINVAL), (dict(rows=0), c2t.EINVAL),
    (dict(vocab=0), c2t.EINVAL), (dict(in_row_stride=992), c2t.EINVAL), (dict(out_row_stride=992, out_dev=2 * A), c2t.EINVAL), (dict(in_seq_stride=-8), c2t.EINVAL),
    (dict(counts_stride=999), c2t.EINVAL), (dict(bias_stride=999), c2t.EINVAL), (dict(allowed_row_stride=-1), c2t.EINVAL), (dict(node_parent_dev=None), c2t.EINVAL),
    (dict(nodes=0), c2t.EINVAL), (dict(out_seq_stride=8000), c2t.EINVAL), (dict(out_row_stride=1008), c2t.EINVAL), (dict(batch=4097), c2t.ERANGE),
    (dict(nodes=8193), c2t.ERANGE), (dict(in_dev=A + 8), c2t.EALIGN), (dict(out_dev=A + 2), c2t.EALIGN), (dict(in_row_stride=1004, out_row_stride=1004), c2t.EALIGN)])
def test_rules_that_are_refused(L, bad, code):
    assert L.c2t_penalize_logits(C.byref(rules(**bad)), None) == code
    assert L.c2t_penalize_logits(None, None) == c2t.EINVAL


def test_counts_that_are_refused(L):
    ok = [A, 1000, 2, 1000, A, 60, A, 7, A, 1, 7, 1, None]
    for at, value, code in ((0, None, c2t.EINVAL), (1, 999, c2t.EINVAL), (2, 0, c2t.EINVAL), (3, 0, c2t.EINVAL), (4, None, c2t.EINVAL), (5, 0, c2t.EINVAL),
                            (7, 6, c2t.EINVAL), (8, None, c2t.EINVAL), (9, 2, c2t.EINVAL), (10, 0, c2t.EINVAL), (2, 4097, c2t.ERANGE)):
        args = list(ok)
        args[at] = value
        assert L.c2t_count_tokens(*args) == code
    args = list(ok)
    args[6], args[10] = None, 61                        # more entries than tokens
    assert L.c2t_count_tokens(*args) == c2t.EINVAL


def test_config_still_refuses_float16_logits():
    s = c2t.Config(batch=1, vocab=100, dtype=c2t.F16, classifier=c2t.CLS_IDENTITY_JOINT)
    assert c2t.c2t_workspace_bytes(s) == 0


def test_packed_structures_have_the_layout_of_c():
    """What a call packs in one step is what the ctypes structures, field by field, say."""
    from paper_2502_13652_b200 import kv_cache as K
    for packed, struct in ((K._ATTENTION, c2t_attention), (K._RULES, c2t_logit_rules)):
        assert packed.size <= C.sizeof(struct) < packed.size + 8
        values = [float(i + 1) / 2 if t is C.c_float else i + 1 for i, (_, t) in enumerate(struct._fields_)]
        got = struct.from_buffer_copy(packed.pack(*values) + bytes(8))
        assert [getattr(got, name) for name, _ in struct._fields_] == values


@pytest.mark.parametrize("what", ["out_seq_stride", "out_token_stride", "out_head_stride"])
def test_rows_in_one_place_are_refused(L, what):
    assert L.c2t_verify_attention(C.byref(cache()), C.byref(attention(**{what: 0})), A, 1 << 40, None) == c2t.EINVAL
    assert L.c2t_penalize_logits(C.byref(rules(in_seq_stride=0, out_seq_stride=0)), None) == c2t.EINVAL


def test_counts_of_more_entries_than_32_bits_reach(L):
    n = (1 << 30) + 1
    assert L.c2t_count_tokens(A, 1000, 2, 1000, A, n, None, 0, A, 0, n, 1, None) == c2t.ERANGE


def test_packed_structures_are_as_long_as_those_of_c():
    """The library copies whole structures: a buffer that ends with the last field is too short for one that ends in padding."""
    from paper_2502_13652_b200 import kv_cache as K
    assert K._ATTENTION.size == C.sizeof(c2t_attention)
    assert K._RULES.size == C.sizeof(c2t_logit_rules)
