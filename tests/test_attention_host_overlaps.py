"""The C entry points of the attention operators refuse outputs over inputs and over themselves, and sizes near 2^31, without a GPU."""
import ctypes

import pytest

import paper_2407_19644_b200 as ubp
from test_attention_host import APPEND, ATTEND, P, cache

D, ROW = 64, 8 * 64          # a row of 4 query heads, 2 key heads and 2 value heads


def call(fn, base, c=None, **at):
    a = list(base)
    a[0] = ctypes.byref(c or cache())
    for i, v in at.items():
        a[int(i[1:])] = v
    return fn(*a)


# place of the queries behind qkv, in elements, and their strides
@pytest.mark.parametrize("place,ts,hs", [(0, 4 * D, D), (0, ROW, 2 * D), (D, ROW, D), (4 * D, ROW, D), (7 * D, ROW, D), (ROW, ROW, D), (-D, ROW, D), (-ROW, ROW, D),
                                         (2 * ROW, 4 * D, D), (8, 4 * D, D)])
def test_queries_over_rows(place, ts, hs):
    assert call(ubp.load().ubp_rotate_append, APPEND, _13=P + 2 * place, _14=ts, _15=hs) == -1


# place of the outputs behind q, in elements
@pytest.mark.parametrize("place,ts,hs", [(0, 4 * D, D), (0, ROW, D), (8, 4 * D, D), (D, 4 * D, D), (-4 * D, 4 * D, D), (8 * D, 4 * D, D), (8 * D, 100 * D, D), (3 * D, 4 * D, 2 * D)])
def test_outputs_over_queries(place, ts, hs):
    assert call(ubp.load().ubp_attention, ATTEND, _11=P + 2 * place, _12=ts, _13=hs) == -1


@pytest.mark.parametrize("ts,hs", [(D, D), (2 * D, D), (3 * D, D), (D, 2 * D), (4 * D - 8, D), (3 * D, 2 * D)])
def test_outputs_over_themselves(ts, hs):
    far = 1 << 30
    assert call(ubp.load().ubp_rotate_append, APPEND, _13=far, _14=ts, _15=hs) == -1
    assert call(ubp.load().ubp_attention, ATTEND, _11=far, _12=ts, _13=hs) == -1


@pytest.mark.parametrize("n", [(1 << 31) - 4096, (1 << 31) - 100, (1 << 31) - 2])
def test_counts_near_the_end_of_32_bits(n):
    L, many, long = ubp.load(), cache(batch=n, starts=P), cache(starts=P)
    far = 1 << 60
    assert call(L.ubp_rotate_append, APPEND, many, _13=far) == -6 and call(L.ubp_rotate_append, APPEND, long, _3=n, _13=far) == -6
    assert call(L.ubp_attention, ATTEND, many, _11=far) == -6 and call(L.ubp_attention, ATTEND, long, _4=n, _11=far) == -6
