"""Attention over a paged cache: which kernel runs, workspaces, long items, captures in a fresh process, extreme arguments."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from attention_ref import BF16, F16, Batch, check

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


def described(b, T=None):
    from paper_2407_19644_b200.binding import _Cache
    s = b.k.stride()
    return _Cache(b.k.data_ptr(), b.v.data_ptr(), s[0], s[1], s[2], b.k.shape[0], b.page, b.Hkv, b.D, 2 if b.dtype == BF16 else 1, b.table.data_ptr(),
                  b.table.stride(0), b.table.shape[1], b.B, b.len_t.data_ptr(), None if b.starts is None else b.starts.data_ptr())


# kernel: 0 = 16 rows an item, steps dealt; 1 = 256 rows; 2 = 16 rows, a cluster an item; and that of the shared prefix (-1: read again)
@pytest.mark.parametrize("new,lengths,Hq,Hkv,max_new,prefix,kernels", [
    ([1, 1], [41, 90], 8, 1, 1, 0, (2, -1)), ([1, 1], [41, 90], 16, 1, 1, 0, (2, -1)), ([1, 1], [41, 90], 17, 1, 1, 0, (1, -1)),
    ([2, 1], [41, 90], 8, 1, 2, 0, (2, -1)), ([3, 1], [41, 90], 8, 1, 3, 0, (1, -1)), ([2, 1], [41, 90], 8, 1, 100, 0, (1, -1)),
    ([1, 1], [70000, 90], 8, 1, 1, 0, (0, -1)), ([1] * 40, [100] * 40, 16, 4, 1, 0, (0, -1)), ([1] * 3, [80, 70, 90], 8, 1, 1, 64, (2, -1)),
    ([5, 1, 1], [80, 70, 90], 8, 1, 5, 64, (1, -1)), ([1] * 3, [150000, 150010, 150020], 8, 2, 1, 150000, (0, 0)),
    ([1] * 40, [9000 + n for n in range(40)], 8, 2, 1, 9000, (0, 1)), ([9] * 30, [9000 + n for n in range(30)], 8, 4, 9, 8960, (1, 1))])
def test_kernel_choice_and_results(ubp, new, lengths, Hq, Hkv, max_new, prefix, kernels):
    b = Batch(new, lengths, Hq, Hkv, 64, F16, 16, prefix=prefix)
    c, k, p = described(b), ctypes.c_int(), ctypes.c_int()
    assert ubp.load().ubp_attention_choice(ctypes.byref(c), b.T, Hq, prefix, max_new, ctypes.byref(k), ctypes.byref(p)) == 0
    assert (k.value, p.value) == kernels
    q = b.queries()
    want, tol = b.exact(q)
    if prefix:
        out = ubp.ubp_prefix_attention(q, *b.args(), prefix, starts=b.starts, max_new=max_new)
    else:
        out = ubp.ubp_attention(q, *b.args(), starts=b.starts, max_new=max_new)
    check(out, want, tol, b.T)
    if max_new > 1 or prefix:
        return
    # more new tokens than the caller says: another kernel would be better, the result is the same
    b = Batch([21, 3, 0, 40], [lengths[0] + 20, 33, 7, 40], Hq, Hkv, 64, F16, 16, behind=1)
    q = b.queries()
    want, tol = b.exact(q, 30, 2)
    check(ubp.ubp_attention(q, *b.args(), starts=b.starts, max_new=1, window=30, sinks=2), want, tol, b.first[-1])


def test_prefix_pages_in_the_first_row_only(ubp):
    """Pages that lie below the prefix as a whole are read through row 0, whichever way the call takes."""
    for lengths, prefix in (([100, 90, 97], 80), ([9000 + n for n in range(40)], 8992)):
        b = Batch([1] * len(lengths), lengths, 8, 2, 64, BF16, 16, prefix=prefix)
        q = b.queries()
        want, tol = b.exact(q)
        b.table[1:, :prefix // 16] = -3
        check(ubp.ubp_prefix_attention(q, *b.args(), prefix, max_new=1), want, tol, b.T)


@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("pad,lead", [(0, 0), (2, 0), (3, 1), (4, 2)])
@pytest.mark.parametrize("prefix", [0, 75000])
def test_workspace_of_the_size_asked_for(ubp, new, pad, lead, prefix):
    """A workspace of exactly that many bytes, between guards; one byte less is refused."""
    b = Batch([new, 1, 1, 1], [new + prefix + 200, prefix + 120, prefix + 1, prefix + 5], 4, 2, 72, BF16, 16, prefix=prefix, wide=600)
    q = b.queries(pad=pad, lead=lead)
    want, tol = b.exact(q)
    c = described(b)
    n = ubp.load().ubp_attention_workspace_size(ctypes.byref(c), q.data_ptr(), q.stride(0), q.stride(1), b.T, 4, 0, 0, prefix, max(new, 1))
    room = torch.full((n + 512,), 77, dtype=torch.uint8, device="cuda")
    fn = ubp.ubp_prefix_attention if prefix else ubp.ubp_attention
    args = (q, *b.args(), prefix) if prefix else (q, *b.args())
    check(fn(*args, starts=b.starts, max_new=new, workspace=room[256:256 + n]), want, tol, b.T)
    assert n > 0 and (room[:256] == 77).all() and (room[256 + n:] == 77).all()
    with pytest.raises(ubp.UbpError) as e:
        fn(*args, starts=b.starts, max_new=new, workspace=room[256:256 + n - 1])
    assert e.value.code == -3
    with pytest.raises(ubp.UbpError) as e:
        fn(*args, starts=b.starts, max_new=new, workspace=room[255:])
    assert e.value.code == -1


def test_items_that_take_milliseconds(ubp):
    """A block may wait for as long as an item takes: eight thousand queries on a million tokens, checked on some rows."""
    n, new, Hq, D, page = 1 << 20, 8192, 4, 64, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(n // page, 1, page, D, device="cuda", generator=g).to(F16) for _ in range(2))
    table = torch.arange(n // page, dtype=torch.int32, device="cuda")[None]
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    q = (4 * torch.randn(new, Hq, D, device="cuda", generator=g)).to(F16)
    out = ubp.ubp_attention(q, k, v, table, lengths, starts=starts)
    ubp.attention_check()
    K, V = k.view(n, D).double(), v.view(n, D).double()
    for t in (0, 1, 63, 64, 4095, 8190, 8191):
        p = n - new + t + 1
        s = (q[t].double() @ K[:p].t()) / 8
        w = torch.softmax(s, 1)
        want, size = w @ V[:p], w @ V[:p].abs()
        # weights rounded to 2^-11 each and errors of the scores (62 exact products, sizes up to 4 * 64 * 4 / 8) as in the other tests
        big = float((q[t].double().abs() @ K[:p].abs().t()).max() / 8)
        tol = size * (2.0 ** -11 + 2 * ((D + 4) * 2.0 ** -23 * big + (big + 16) * 2.0 ** -21)) + 2.0 ** -11 * want.abs() + 2.0 ** -24
        # sums of a million weights, a few of which matter: the partial sums' roundings add to at most 2^-23 of the sum for each of
        # a tile's 128 and of the 8192 tiles that a row is rescaled or added over
        tol += size * 2 * (128 + 8192) * 2.0 ** -23 + 2.0 ** -25 * float(V.abs().mean()) * p * float(w.max())
        assert ((out[t].double() - want).abs() <= tol).all()


def test_first_call_of_a_process_is_captured():
    code = """
import torch, paper_2407_19644_b200 as ubp
q = torch.randn(2, 4, 64, device='cuda').bfloat16()
k, v = (torch.randn(8, 2, 16, 64, device='cuda').bfloat16() for _ in range(2))
t = torch.arange(8, dtype=torch.int32, device='cuda').view(2, 4)
n = torch.tensor([60, 33], dtype=torch.int32, device='cuda')
o, p = torch.zeros(2, 4, 64, device='cuda').bfloat16(), torch.zeros(2, 4, 64, device='cuda').bfloat16()
s = torch.tensor([0, 1, 2], dtype=torch.int32, device='cuda')
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    ubp.ubp_attention(q, k, v, t, n, out=o)
    ubp.ubp_attention(q, k, v, t, n, out=p, starts=s, max_new=50)
    ubp.ubp_prefix_attention(q, k, v, t, n, 16)
    ubp.ubp_rotate_append(torch.zeros(2, 8 * 64, device='cuda').bfloat16(), 4, k.clone(), v.clone(), t, n)
g.replay()
torch.cuda.synchronize()
a = ubp.ubp_attention(q, k, v, t, n)
assert torch.equal(o, a) and (p.float() - a.float()).abs().max() < 0.05, (o - a).abs().max()
print('captured ok')
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured ok" in r.stdout, r.stdout[-1000:] + r.stderr[-2000:]


@pytest.mark.parametrize("max_new", [1, 60])
def test_extreme_windows(ubp, max_new):
    most = (1 << 31) - 1
    b = Batch([1, 2], [300, 1], 4, 2, 64, BF16, 16)          # (the second has more new tokens than it is long)
    b.K[1], b.V[1] = b.K[1][:1], b.V[1][:1]
    q = b.queries()
    out = ubp.ubp_attention(q, *b.args(), starts=b.starts, max_new=max_new)
    for window, sinks in ((most, 0), (most, most), (5, most), (300, 300)):
        got = ubp.ubp_attention(q, *b.args(), starts=b.starts, window=window, sinks=sinks, max_new=max_new)
        assert torch.isfinite(got).all() and ((got.float() - out.float()).abs() <= 2.0 ** -7 * out.float().abs() + 2.0 ** -7).all()
    got = ubp.ubp_attention(q, *b.args(), starts=b.starts, window=1, max_new=max_new)     # itself only: its own value
    assert torch.equal(got[0], b.V[0][299].repeat_interleave(2, 0)) and (got[1] == 0).all() and torch.equal(got[2], b.V[1][0].repeat_interleave(2, 0))


@pytest.mark.parametrize("max_new", [1, 60])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_unseen_tokens_do_not_matter(ubp, max_new, value):
    """Keys and values that no new token sees -- behind the lengths, outside windows, before a page's first seen token -- may be
    anything; so may unused pages."""
    for window, sinks in ((0, 0), (100, 5), (37, 130)):
        b = Batch([1, 1, 1], [437, 128, 1], 4, 2, 128, BF16, 64, seed=window)
        q = b.queries()
        want, tol = b.exact(q, window, sinks)
        hidden = [torch.arange(n, device="cuda") for n in b.lengths]
        for s, n in enumerate(b.lengths):
            j = hidden[s]
            gone = (j <= n - 1 - window) & (j >= sinks) if window else j < 0
            page, slot = b.table[s].long()[j[gone] // 64], j[gone] % 64
            b.k[page, :, slot] = value
            b.v[page, :, slot] = value
        check(ubp.ubp_attention(q, *b.args(), starts=b.starts, window=window, sinks=sinks, max_new=max_new), want, tol, 3)


def test_results_do_not_depend_on_neighbours(ubp):
    """A sequence's result is the same to its rounding alone and in a batch."""
    b = Batch([3, 70, 1, 200], [90, 700, 1300, 200], 6, 2, 96, BF16, 32)
    q = b.queries()
    want, tol = b.exact(q)
    for s in range(4):
        rows = slice(b.first[s], b.first[s + 1])
        alone = torch.tensor([0, b.new[s]], dtype=torch.int32, device="cuda")
        out = ubp.ubp_attention(q[rows], b.k, b.v, b.table[s:s + 1], b.len_t[s:s + 1], starts=alone)
        check(out, want[rows], tol[rows], b.new[s])


@pytest.mark.parametrize("D,G,Hkv,new,dtype", [
    (64, 1, 2, [1] * 9, F16), (128, 4, 1, [1] * 9, BF16), (80, 16, 2, [1, 3, 0, 1, 40, 1, 1, 1, 2], F16), (72, 40, 2, [1] * 9, BF16),
    (128, 1, 1, [1] * 9, BF16), (96, 3, 3, [30, 2, 70, 1, 1, 0, 200, 1, 1], BF16)])
def test_prefix_read_once(ubp, D, G, Hkv, new, dtype):
    """A prefix long enough for a call of its own, ending inside a page, queries inside it among others."""
    prefix = 120 * 10 ** 6 // (8 * Hkv * D * 4) + 13
    lengths = [prefix + [40, 3, 0, 1, 200, 700, 129, 64, 2][s] for s in range(9)]
    b = Batch(new, lengths, Hkv * G, Hkv, D, dtype, 64, prefix=prefix, behind=2, seed=D)
    q = b.queries(pad=G % 2)
    c, k, p = described(b), ctypes.c_int(), ctypes.c_int()
    assert ubp.load().ubp_attention_choice(ctypes.byref(c), b.T, Hkv * G, prefix, max(new), ctypes.byref(k), ctypes.byref(p)) == 0 and p.value >= 0
    for window, sinks in ((0, 0), (500, 5)):
        want, tol = b.exact(q, window, sinks)
        out = torch.full((b.T, Hkv * G, D), -77.0, dtype=dtype, device="cuda")
        got = ubp.ubp_prefix_attention(q, *b.args(), prefix, starts=b.starts, max_new=max(new), window=window, sinks=sinks, out=out)
        check(got, want, tol, b.first[-1])
        assert (out[b.first[-1]:] == -77.0).all()
        again = ubp.ubp_prefix_attention(q, *b.args(), prefix, starts=b.starts, max_new=max(new), window=window, sinks=sinks, out=torch.empty_like(out))
        assert torch.equal(again[:b.first[-1]], out[:b.first[-1]])


@pytest.mark.parametrize("G", [3, 5, 48, 127])
def test_unused_rows_have_no_say(ubp, G):
    """Groups that do not fill a tile of 128 rows: what its other rows hold does not move a bit of the result."""
    b = Batch([90, 33], [700, 1500], G, 1, 64, BF16, 16)
    q = b.queries(3.0)
    first = ubp.ubp_attention(q, *b.args(), starts=b.starts)
    want, tol = b.exact(q)
    check(first, want, tol, b.T)
    other = Batch([300], [300], 8, 1, 128, BF16, 16, seed=3)
    for scale in (1e-3, 1.0, 100.0):
        ubp.ubp_attention(other.queries(scale), *other.args(), starts=other.starts)       # leaves its queries in the SMs' memory
        assert torch.equal(ubp.ubp_attention(q, *b.args(), starts=b.starts), first)


@pytest.mark.parametrize("D,G,Hkv,new", [(128, 4, 1, [1] * 9), (64, 3, 2, [1, 3, 0, 1, 200, 1, 1, 1, 2])])
def test_prefix_under_a_window(ubp, D, G, Hkv, new):
    """Windows that leave enough of a prefix for a call of its own, and shorter ones, under which each sequence reads its own part."""
    prefix = 120 * 10 ** 6 // (8 * Hkv * D * 4) + 2000
    lengths = [prefix + [40, 3, 0, 1, 200, 700, 129, 64, 2][s] for s in range(9)]
    b = Batch(new, lengths, Hkv * G, Hkv, D, BF16, 64, prefix=prefix, seed=D)
    q, c = b.queries(), described(b)
    size = lambda window: ubp.load().ubp_attention_workspace_size(ctypes.byref(c), q.data_ptr(), q.stride(0), q.stride(1), b.T, Hkv * G, window, 0, prefix, max(new))
    assert size(prefix - 100) > b.T * Hkv * G * D * 4 + size(100)        # (a call of its own leaves a row of sums for each query)
    for window, sinks in ((prefix - 100, 3), (prefix + 50, 0), (prefix // 2, 70), (100, 70)):
        want, tol = b.exact(q, window, sinks)
        check(ubp.ubp_prefix_attention(q, *b.args(), prefix, starts=b.starts, max_new=max(new), window=window, sinks=sinks), want, tol, b.T)


@pytest.mark.parametrize("new,old,window,prefix,whole", [
    ([1, 5, 0, 300, 90, 2] * 4, [0, 700, 30, 400, 1, 90] * 4, 0, 0, True), ([200, 31, 600], [1000, 1500, 936], 0, 0, True),
    ([200, 31, 600], [1000, 1700, 936], 0, 0, False), ([1500, 1, 0, 700], [0, 9000, 3, 20], 1000, 0, True), ([3] * 7, [1, 9, 300, 0, 2, 30, 31], 0, 70000, True),
    ([1] * 150, [n * 17 % 600 for n in range(150)], 0, 0, True), ([1] * 400, [n * 13 % 700 for n in range(400)], 0, 0, True),
    ([1] * 60, [1900] * 60, 0, 0, False), ([1] * 70, [n * 170 for n in range(70)], 300, 0, True), ([1] * 40, [n * 9 for n in range(40)], 0, 20000, True)])
def test_short_items_are_not_cut(ubp, new, old, window, prefix, whole):
    """Calls of short items need no partial results: their blocks take whole items, wherever the lengths put the shares' ends."""
    b = Batch(new, [prefix + n + o for n, o in zip(new, old)], 8, 2, 128, BF16, 32, seed=len(new), prefix=prefix, behind=0 if max(new) == 1 else 2, single=max(new) == 1)
    q = b.queries()
    c = described(b)
    size = lambda sinks, w: ubp.load().ubp_attention_workspace_size(ctypes.byref(c), q.data_ptr(), q.stride(0), q.stride(1), b.T, 8, w, sinks, prefix, max(new))
    if not prefix:
        assert (size(0, window) == 0) == whole
    for sinks in (0, 3) if window else (0,):
        want, tol = b.exact(q, window, sinks)
        fn, args = (ubp.ubp_prefix_attention, b.args() + (prefix,)) if prefix else (ubp.ubp_attention, b.args())
        out = torch.full((b.T, 8, 128), -77.0, dtype=BF16, device="cuda")
        fn(q, *args, starts=b.starts, window=window, sinks=sinks, max_new=max(new), out=out)
        check(out, want, tol, b.first[-1])
        assert (out[b.first[-1]:] == -77.0).all()
        again = fn(q, *args, starts=b.starts, window=window, sinks=sinks, max_new=max(new), out=torch.full_like(out, -77.0))
        assert torch.equal(again, out)
