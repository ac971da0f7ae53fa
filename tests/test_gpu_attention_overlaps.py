"""Outputs that lie over inputs, or over themselves: refused where rows would be read after they were written, allowed otherwise."""
import ctypes

import pytest
import torch

from attention_ref import BF16, Batch
from test_gpu_attention_paths import described

pytestmark = pytest.mark.gpu

HQ, HKV, D = 4, 2, 64


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


def buffer(b, cols):
    return torch.randn(b.T, cols, generator=b.g, device="cuda").to(b.dtype)


def code_of(ubp, f):
    with pytest.raises((ubp.UbpError, ValueError)) as e:
        f()
    return e.value.code if isinstance(e.value, ubp.UbpError) else -1


@pytest.mark.parametrize("pad", [0, 3])
def test_append_refuses_queries_over_rows(ubp, pad):
    b = Batch([70, 30], [70, 40], HQ, HKV, D, BF16, 16)
    width = (HQ + 2 * HKV) * D
    whole = buffer(b, width + pad)
    qkv = whole[:, :width]
    heads = lambda start, ts, hs: whole.view(-1)[start:].as_strided((b.T, HQ, D), (ts, hs, 1))
    keep = whole.clone(), b.k.clone().view(torch.int16)
    for out in (heads(0, HQ * D, D), heads(0, width + pad, 2 * D), heads(D, width + pad, D), heads(HQ * D, width + pad, D), heads(HQ * D, HQ * D, D)):
        assert code_of(ubp, lambda: ubp.ubp_rotate_append(qkv, HQ, *b.args(), starts=b.starts, out=out)) == -1
    less = torch.tensor([0, 70, 99], dtype=torch.int32, device="cuda")
    up = whole[1:, :HQ * D].unflatten(1, (HQ, D))              # the queries' places of the rows behind
    assert code_of(ubp, lambda: ubp.ubp_rotate_append(qkv[:-1], HQ, *b.args(), starts=less, out=up)) == -1
    assert torch.equal(whole, keep[0]) and torch.equal(b.k.view(torch.int16), keep[1])
    with pytest.raises(ValueError):
        ubp.ubp_rotate_append(qkv, HQ, *b.args(), starts=b.starts, out=heads(0, HQ * D, D))
    one = Batch([1], [5], HQ, HKV, D, BF16, 16)                # a single token: heads over other heads
    row = buffer(one, width)
    assert code_of(ubp, lambda: ubp.ubp_rotate_append(row, HQ, *one.args(), out=row.view(-1).as_strided((1, HQ, D), (width, 2 * D, 1)))) == -1


def test_append_allows_what_lies_apart(ubp):
    b = Batch([70, 30], [70, 40], HQ, HKV, D, BF16, 16)
    width, rot = (HQ + 2 * HKV) * D, ubp.rotation_table(100, D)
    whole = buffer(b, width + HQ * D)
    run = lambda qkv, out=None: ubp.ubp_rotate_append(qkv, HQ, *b.args(), starts=b.starts, rotation=rot, out=out)
    want = run(whole[:, :width].clone())
    beside = whole.clone()                                     # in columns of the same rows, before and behind
    assert torch.equal(run(beside[:, :width], beside[:, width:].unflatten(1, (HQ, D))), want) and torch.equal(beside[:, :width], whole[:, :width])
    front = torch.cat([whole[:, width:], whole[:, :width]], 1)
    assert torch.equal(run(front[:, HQ * D:], front[:, :HQ * D].unflatten(1, (HQ, D))), want)
    own = whole.clone()                                        # in the queries' own place
    assert torch.equal(run(own[:, :width], own[:, :HQ * D].unflatten(1, (HQ, D))), want)
    flat = torch.cat([whole[:, :width].reshape(-1), whole.new_zeros(b.T * HQ * D)])      # one behind the other
    assert torch.equal(run(flat[:b.T * width].view(b.T, width), flat[b.T * width:].view(b.T, HQ, D)), want)
    outside = torch.empty(HQ, b.T, D, dtype=BF16, device="cuda")                          # heads outside tokens
    assert torch.equal(run(whole[:, :width].clone(), outside.transpose(0, 1)), want)


def c_attention(ubp, b, q, out, room):
    c = described(b)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    stride = lambda t: (t.stride(0), t.stride(1))
    return ubp.load().ubp_attention(ctypes.byref(c), ptr(q), *stride(q), b.T, HQ, 0.125, 0, 0, 0, b.T, ptr(out), *stride(out), ptr(room), room.numel(),
                                    ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))


def test_attention_refuses_outputs_over_queries(ubp):
    b = Batch([70, 30], [170, 40], HQ, HKV, D, BF16, 16)
    whole = buffer(b, 2 * HQ * D)
    room = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    heads = lambda start, ts, hs: whole.view(-1)[start:].as_strided((b.T, HQ, D), (ts, hs, 1))
    q, keep = heads(0, 2 * HQ * D, D), whole.clone()
    for out in (q, heads(8, 2 * HQ * D, D), heads(D, 2 * HQ * D, D), heads(0, HQ * D, D), heads(0, 2 * HQ * D, 2 * D), heads(D, 2 * HQ * D, 2 * D),
                heads(D // 2, 2 * HQ * D, 2 * D)):
        assert c_attention(ubp, b, q, out, room) == -1
        assert code_of(ubp, lambda: ubp.ubp_attention(q, *b.args(), starts=b.starts, out=out)) == -1
    assert torch.equal(whole, keep)


def test_attention_allows_outputs_beside_queries(ubp):
    b = Batch([70, 30], [170, 40], HQ, HKV, D, BF16, 16)
    whole = buffer(b, 2 * HQ * D)
    pairs = lambda x: (x[:, :HQ * D].unflatten(1, (HQ, D)), x[:, HQ * D:].unflatten(1, (HQ, D)))            # side by side, either first
    turns = lambda x: x.view(b.T, HQ, 2, D).unbind(2)                                                        # head by head
    outer = lambda x: x.view(2 * HQ, b.T, D).transpose(0, 1).split(HQ, 1)                                    # heads outside tokens
    behind = lambda x: x.view(2 * b.T, HQ, D).split(b.T)
    for layout in (pairs, turns, outer, behind):
        for first in (0, 1):
            x = whole.clone()
            q, out = layout(x)[first], layout(x)[1 - first]
            want = ubp.ubp_attention(q.clone(memory_format=torch.contiguous_format), *b.args(), starts=b.starts)
            before = q.clone()
            assert torch.equal(ubp.ubp_attention(q, *b.args(), starts=b.starts, out=out), want) and torch.equal(q, before)


def test_outputs_over_themselves(ubp):
    """Heads that share places with the heads of other tokens."""
    b = Batch([70, 30], [170, 40], HQ, HKV, D, BF16, 16)
    qkv, q = buffer(b, (HQ + 2 * HKV) * D), b.queries()
    buf = torch.full((1 << 17,), 5.0, dtype=BF16, device="cuda")
    for ts, hs in ((D, D), (2 * D, D), (3 * D, D), (D, 2 * D), (3 * D, 2 * D), (4 * D - 8, D), (D, 99 * D), (8 * D, 4 * D + 8)):
        out = buf.as_strided((b.T, HQ, D), (ts, hs, 1))
        assert code_of(ubp, lambda: ubp.ubp_rotate_append(qkv, HQ, *b.args(), starts=b.starts, out=out)) == -1
        assert code_of(ubp, lambda: ubp.ubp_attention(q, *b.args(), starts=b.starts, out=out)) == -1
    assert (buf == 5.0).all()
    want = ubp.ubp_attention(q, *b.args(), starts=b.starts)
    for ts, hs in ((4 * D, D), (D, 100 * D), (9 * D, 2 * D), (2 * D, 201 * D), (8 * D, 4 * D + 32)):
        assert torch.equal(ubp.ubp_attention(q, *b.args(), starts=b.starts, out=buf.as_strided((b.T, HQ, D), (ts, hs, 1))), want)
