"""The C entry points of the attention operators: refusals and workspace, without a GPU."""
import ctypes

import pytest

import paper_2407_19644_b200 as ubp
from paper_2407_19644_b200.binding import _Cache

P = 1 << 20      # (never dereferenced)


def cache(**kw):
    d = dict(k=P, v=P, page_stride=2 * 16 * 64, head_stride=16 * 64, token_stride=64, pages=10, page_size=16, kv_heads=2, head_dim=64, dtype=2,
             table=P, table_stride=4, table_width=4, batch=3, lengths=P, starts=None)
    d.update(kw)
    return _Cache(*[d[f[0]] for f in _Cache._fields_])


BAD = [(dict(k=None), -1), (dict(v=None), -1), (dict(k=P + 8), -1), (dict(v=P + 2), -1), (dict(page_stride=2 * 16 * 64 + 4), -1), (dict(head_stride=63), -1),
       (dict(head_stride=56), -1), (dict(token_stride=56), -1), (dict(token_stride=65), -1), (dict(page_stride=0), -1), (dict(pages=0), -1),
       (dict(pages=1 << 31), -6), (dict(page_size=0), -1), (dict(page_size=4), -6), (dict(page_size=24), -6), (dict(kv_heads=0), -1), (dict(kv_heads=3), -1),
       (dict(head_dim=0), -1), (dict(head_dim=60), -6), (dict(head_dim=136), -6), (dict(dtype=0), -1), (dict(dtype=3), -1), (dict(dtype=9), -1), (dict(table=None), -1),
       (dict(table=P + 1), -1), (dict(table_stride=3), -1), (dict(table_width=0), -1), (dict(batch=4), -1), (dict(batch=-1), -1), (dict(lengths=None), -1),
       (dict(lengths=P + 2), -1), (dict(starts=P + 2), -1), (dict(batch=(1 << 31) - 1, starts=P), -6)]

#            cache  qkv  ld       T  heads  gammas      eps   rotation          rotated   q        strides   stream
APPEND = [None, P, 8 * 64, 3, 4, None, None, 1e-6, P, 64, 100, 64, 0, P, 4 * 64, 64, None]
#            cache  q    strides      T  heads  scale window sinks prefix max_new  out  strides   workspace  bytes    stream
ATTEND = [None, P, 4 * 64, 64, 3, 4, 0.125, 0, 0, 0, 1, P, 4 * 64, 64, P, 1 << 40, None]


@pytest.mark.parametrize("change,code", BAD)
def test_bad_caches(change, code):
    L, c = ubp.load(), cache(**change)
    assert L.ubp_rotate_append(ctypes.byref(c), *APPEND[1:]) == code
    assert L.ubp_attention(ctypes.byref(c), *ATTEND[1:]) == code
    assert L.ubp_attention_workspace_size(ctypes.byref(c), P, 4 * 64, 64, 3, 4, 0, 0, 0, 1) == 0


def refused(fn, base, changes):
    c = cache()
    for at, v, code in changes:
        a = list(base)
        a[0] = ctypes.byref(c)
        a[at] = v
        assert fn(*a) == code, (at, v)


def test_append_refusals():
    nan = float("nan")
    refused(ubp.load().ubp_rotate_append, APPEND,
            [(0, None, -1), (1, None, -1), (1, P + 1, -1), (2, 8 * 64 - 1, -1), (3, -1, -1), (4, 0, -1), (4, 3, -1), (5, P + 1, -1), (6, P + 1, -1), (7, -1.0, -1),
             (7, nan, -1), (8, P + 2, -1), (9, 63, -1), (10, 0, -1), (11, 0, -1), (11, 63, -1), (11, 66, -1), (13, None, -1), (13, P + 1, -1), (14, 63, -1),
             (15, 63, -1), (3, 1 << 31, -1)])


def test_attention_refusals():
    nan, inf = float("nan"), float("inf")
    refused(ubp.load().ubp_attention, ATTEND,
            [(0, None, -1), (1, None, -1), (1, P + 1, -1), (2, 63, -1), (3, 63, -1), (4, -1, -1), (5, 3, -1), (6, 0.0, -1), (6, -1.0, -1), (6, nan, -1), (6, inf, -1),
             (7, -1, -1), (8, -1, -1), (9, -1, -1), (9, 65, -1), (10, 0, -1), (11, None, -1), (11, P + 1, -1), (12, 63, -1), (13, 63, -1)])


def test_no_tokens_is_a_no_op():
    L, c = ubp.load(), cache(batch=0, k=None, table=None)
    a = list(ATTEND)
    a[0], a[1], a[4] = ctypes.byref(c), None, 0
    assert L.ubp_attention(*a) == 0
    a = list(APPEND)
    a[0], a[1], a[3] = ctypes.byref(c), None, 0
    assert L.ubp_rotate_append(*a) == 0
    assert L.ubp_attention_workspace_size(ctypes.byref(c), None, 4 * 64, 64, 0, 4, 0, 0, 0, 1) == 0
