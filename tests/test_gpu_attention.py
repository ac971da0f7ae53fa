"""Attention over a paged cache against the formula in 64 bits: head layouts, pages, lengths, windows, strides."""
import pytest
import torch

from attention_ref import BF16, F16, Batch, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


HEADS = [(1, 1, 64), (3, 1, 80), (4, 2, 128), (8, 1, 8), (32, 4, 128), (48, 3, 72), (20, 1, 96), (32, 1, 120), (136, 1, 64), (258, 2, 16)]
NEW = [
    ([1], [1]), ([1], [300]), ([1, 1, 1], [17, 1000, 129]), ([1] * 7, [0, 1, 8, 128, 2049, 640, 127]),       # a token each
    ([5], [5]), ([130], [130]), ([300], [777]), ([0, 3, 0, 257, 1, 64, 0], [9, 3, 0, 300, 513, 64, 40]),      # prompts and continuations
    ([40, 17], [1200, 17])]
WINDOWS = [(0, 0), (1, 0), (100, 3), (128, 130), (500, 1)]


def run(ubp, b, q, fn="ubp_attention", **kw):
    out = torch.full((b.T, b.Hq, b.D), -77.0, dtype=b.dtype, device="cuda")
    kw.setdefault("starts", b.starts)
    got = getattr(ubp, fn)(q, *b.args(), out=out, **kw)
    assert got is out
    assert (out[b.first[-1]:] == -77.0).all()                  # rows of no sequence
    return out


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("case", range(len(NEW)))
def test_heads_and_lengths(ubp, dtype, Hq, Hkv, D, case):
    new, lengths = NEW[case]
    single = all(n == 1 for n in new)
    b = Batch(new, lengths, Hq, Hkv, D, dtype, [16, 8, 64, 128, 32][(case + D) % 5], seed=case + D, behind=0 if single else 3, single=single)
    q = b.queries()
    for window, sinks in ((0, 0), WINDOWS[1 + (case + Hq) % 4]):
        want, tol = b.exact(q, window, sinks)
        check(run(ubp, b, q, window=window, sinks=sinks), want, tol, b.first[-1])
        if single or max(new) <= 5:
            check(run(ubp, b, q, window=window, sinks=sinks, max_new=max(new)), want, tol, b.first[-1])


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("new,lengths", [([1, 1], [1500, 90]), ([700], [700]), ([70, 300], [1000, 411])])
def test_windows(ubp, window, sinks, new, lengths):
    b = Batch(new, lengths, 6, 2, 64, BF16, 16, seed=window + 1)
    q = b.queries(3.0)
    want, tol = b.exact(q, window, sinks, 0.3)
    check(run(ubp, b, q, window=window, sinks=sinks, scale=0.3), want, tol, b.first[-1])


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256, 1024])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("new", [1, 150])
def test_pages_and_layouts(ubp, page, layout, new):
    b = Batch([new, new], [1030, 151], 4, 2, 72, F16, page, seed=page, layout=layout, wide=3)
    q = b.queries(pad=5, lead=1)                                # nothing aligned
    want, tol = b.exact(q)
    check(run(ubp, b, q), want, tol, b.first[-1])


def test_strided_output_and_queries(ubp):
    b = Batch([1, 40, 3], [300, 40, 1029], 6, 3, 80, BF16, 16)
    q = b.queries(pad=3, lead=1)
    want, tol = b.exact(q)
    for pad in (1, 8):
        buf = torch.full((b.T, 6, 80 + pad), 5.0, dtype=BF16, device="cuda")
        ubp.ubp_attention(q, *b.args(), starts=b.starts, out=buf[:, :, :80])
        check(buf[:, :, :80], want, tol, b.T)
        assert (buf[:, :, 80:] == 5.0).all()
    flat = torch.empty(6, b.T, 80, dtype=BF16, device="cuda")   # heads outside tokens
    with pytest.raises(ValueError):
        ubp.ubp_attention(q, *b.args(), starts=b.starts, out=flat.transpose(0, 1)[:, :, :79])
    ubp.ubp_attention(q, *b.args(), starts=b.starts, out=flat.transpose(0, 1))
    check(flat.transpose(0, 1), want, tol, b.T)


@pytest.mark.parametrize("D,G", [(64, 1), (128, 4), (128, 16), (80, 40)])
@pytest.mark.parametrize("own", [[1, 1, 1], [1, 30, 700, 1, 2, 90], [1] * 70])
@pytest.mark.parametrize("prefix", [1, 16, 129, 1001])
def test_prefix(ubp, D, G, own, prefix):
    b = Batch([1] * len(own), [prefix + n for n in own], 2 * G, 2, D, BF16 if D == 128 else F16, 16, seed=prefix, prefix=prefix)
    q = b.queries()
    for window, sinks in ((0, 0), (300, 5)):
        want, tol = b.exact(q, window, sinks)
        check(run(ubp, b, q, "ubp_prefix_attention", prefix=prefix, max_new=1, window=window, sinks=sinks), want, tol, b.T)


def test_prefix_with_prompts(ubp):
    """Several new tokens a sequence, some of them inside the prefix; rows behind the last sequence."""
    b = Batch([3, 200, 0, 1], [300, 410, 300, 301], 8, 2, 64, BF16, 32, prefix=300, behind=2)
    q = b.queries()
    want, tol = b.exact(q)
    check(run(ubp, b, q, "ubp_prefix_attention", prefix=300), want, tol, b.first[-1])


def test_rows_that_see_nothing(ubp):
    """Sequences without tokens, and more new tokens than the sequence has."""
    b = Batch([1, 4, 2], [0, 2, 0], 4, 2, 64, BF16, 16)
    q = b.queries()
    out = run(ubp, b, q)
    assert (out[0] == 0).all() and (out[1:3] == 0).all() and (out[5:] == 0).all()
    v = b.V[1].double()
    assert torch.equal(out[3].double(), v[0].repeat_interleave(2, 0))      # one key seen: its value
    out = run(ubp, b, q, "ubp_prefix_attention", prefix=16)
    assert (out[0] == 0).all() and (out[1:3] == 0).all() and (out[5:] == 0).all()


def test_numbers_that_make_no_sense(ubp):
    """Pages outside the cache read as zeros; lengths and starts are cut."""
    b = Batch([1, 1], [40, 40], 2, 1, 64, F16, 16)
    q = b.queries()
    for bad in (-1, 1 << 30, b.k.shape[0]):
        b.table[1, 1] = bad
        b.K[1][16:32] = 0
        b.V[1][16:32] = 0
        want, tol = b.exact(q)
        check(run(ubp, b, q), want, tol, 2)
        check(run(ubp, b, q, max_new=100), want, tol, 2)
    b.len_t[0] = -5
    assert (run(ubp, b, q)[0] == 0).all()
    b = Batch([2, 3], [40, 48], 2, 1, 64, F16, 16)
    q = b.queries()
    want, tol = b.exact(q)
    b.len_t[1] = 1 << 30                                        # cut to the table's 48 tokens
    check(run(ubp, b, q), want, tol, 5)
    b.starts[2] = 1 << 30                                       # cut to the 5 rows
    check(run(ubp, b, q), want, tol, 5)
    b.starts[1] = -4                                            # no rows for the first sequence, all five for the second
    out = run(ubp, b, q)
    assert torch.isfinite(out).all()


def test_special_values(ubp):
    b = Batch([1, 1, 1], [200, 300, 150], 4, 2, 64, BF16, 16)
    q = b.queries()
    want, tol = b.exact(q)
    q[1, 0, 3] = float("nan")
    b.v[b.table[2, 3].long(), 1, 5, 7] = float("inf")
    out = run(ubp, b, q)
    ok = torch.ones(3, 4, dtype=torch.bool, device="cuda")
    ok[1, 0] = ok[2, 2:] = False
    assert out[1, 0].isnan().all() and (~torch.isfinite(out[2, 2:, 7])).all()
    assert ((out.double() - want).abs() <= tol)[ok].all()
    # large scores: nothing overflows, and the largest key's value is the result
    q = b.queries(300.0)
    b.write()
    want, tol = b.exact(q)
    check(run(ubp, b, q), want, tol, 3)


def test_no_rows(ubp):
    b = Batch([0, 0], [5, 0], 4, 2, 64, BF16, 16)
    q = torch.empty(0, 4, 64, dtype=BF16, device="cuda")
    assert ubp.ubp_attention(q, *b.args(), starts=b.starts).shape == (0, 4, 64)
    q = torch.full((3, 4, 64), 2.0, dtype=BF16, device="cuda")             # rows, but of no sequence
    out = torch.full_like(q, 3.0)
    ubp.ubp_attention(q, *b.args(), starts=b.starts, out=out)
    assert (out == 3.0).all()


def test_many_sequences(ubp):
    """More sequences than a block has threads, empty ones among them."""
    n = 700
    new = [(b * 7 % 5) // 2 for b in range(n)]
    lengths = [a + b * 13 % 90 for b, a in enumerate(new)]
    b = Batch(new, lengths, 4, 1, 64, BF16, 16)
    q = b.queries()
    want, tol = b.exact(q, 40, 2)
    check(run(ubp, b, q, window=40, sinks=2), want, tol, b.T)
    check(run(ubp, b, q, window=40, sinks=2, max_new=2), want, tol, b.T)


def test_offsets_beyond_32_bits(ubp):
    """A cache of 5 10^9 values whose last pages are in use."""
    pages, page, Hkv, D = 4900, 64, 128, 128
    k = torch.empty(pages, Hkv, page, D, dtype=BF16, device="cuda")
    v = torch.empty_like(k)
    assert k.numel() > 1 << 32
    b = Batch([1, 150], [200, 150], Hkv, Hkv, D, BF16, page)
    n = b.k.shape[0]
    k[-n:], v[-n:] = b.k, b.v
    q = b.queries()
    want, tol = b.exact(q)
    out = ubp.ubp_attention(q, k, v, torch.where(b.table >= 0, b.table + (pages - n), b.table), b.len_t, starts=b.starts)
    check(out, want, tol, b.T)


def test_reproducible_and_captured(ubp):
    """Equal results from call to call; a captured call follows the lengths, and two graphs may take turns on one workspace."""
    b = Batch([1, 1, 1], [900, 33, 2000], 8, 2, 128, BF16, 16, single=True)
    q = b.queries()
    first = run(ubp, b, q, starts=None)
    for _ in range(5):
        assert torch.equal(run(ubp, b, q, starts=None), first)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.zeros_like(first) for _ in range(2)], []
    for i, o in enumerate(outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ubp.ubp_attention(q, *b.args(), window=0 if i == 0 else 64, out=o, workspace=ws)
        graphs.append(g)
    lengths = b.lengths
    for change in (lengths, [5, 33, 1999], lengths):
        b.len_t.copy_(torch.tensor(change, dtype=torch.int32))
        graphs[0].replay()
        graphs[1].replay()
        b.lengths, keep = change, (b.K, b.V)
        b.K, b.V = [x[:n] for x, n in zip(b.K, change)], [x[:n] for x, n in zip(b.V, change)]
        for o, window in zip(outs, (0, 64)):
            want, tol = b.exact(q, window)
            check(o, want, tol, 3)
        b.K, b.V = keep


def test_streams(ubp):
    """Two streams at once, each with a workspace of its own."""
    cases = [Batch([1, 1], [3000, 100], 8, 2, 128, BF16, 16, seed=1), Batch([200], [900], 4, 1, 64, F16, 32, seed=2)]
    qs = [b.queries() for b in cases]
    want = [b.exact(q) for b, q in zip(cases, qs)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):
        for i, (b, q, s) in enumerate(zip(cases, qs, streams)):
            outs[i].append(ubp.ubp_attention(q, *b.args(), starts=b.starts, stream=s))
    torch.cuda.synchronize()
    for i, b in enumerate(cases):
        for o in outs[i]:
            check(o, *want[i], b.T)


def test_refusals(ubp):
    b = Batch([1, 1], [40, 40], 4, 2, 64, BF16, 16)
    q = b.queries()
    k, v, t, n = b.args()
    bad = [lambda: ubp.ubp_attention(q[:, :3], k, v, t, n), lambda: ubp.ubp_attention(q.half(), k, v, t, n), lambda: ubp.ubp_attention(q[:1], k, v, t, n),
           lambda: ubp.ubp_attention(q, k, v[:1], t, n), lambda: ubp.ubp_attention(q, k, v.half(), t, n), lambda: ubp.ubp_attention(q, k, v, t.long(), n),
           lambda: ubp.ubp_attention(q, k, v, t, n[:1]), lambda: ubp.ubp_attention(q, k, v, t, n.long()), lambda: ubp.ubp_attention(q, k, v, t, n, starts=n),
           lambda: ubp.ubp_attention(q.cpu(), k, v, t, n), lambda: ubp.ubp_attention(q, k.cpu(), v.cpu(), t, n), lambda: ubp.ubp_attention(q, k, v, t, n, out=q),
           lambda: ubp.ubp_attention(q, k, v, t, n, out=torch.empty(2, 4, 63, device="cuda", dtype=BF16)), lambda: ubp.ubp_attention(q, k, v, t, n, window=-1),
           lambda: ubp.ubp_attention(q, k, v, t, n, sinks=1 << 40), lambda: ubp.ubp_attention(q, k.float(), v.float(), t, n),
           lambda: ubp.ubp_attention(q, k.transpose(2, 3), v.transpose(2, 3), t, n)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    k7, v7 = (torch.zeros(3, 2, 12, 64, device="cuda", dtype=BF16) for _ in range(2))
    k9, v9 = (torch.zeros(3, 2, 16, 60, device="cuda", dtype=BF16) for _ in range(2))
    q9 = torch.zeros(2, 4, 60, device="cuda", dtype=BF16)
    ko, vo = (torch.zeros(3, 2, 16, 68, device="cuda", dtype=BF16)[..., :64] for _ in range(2))
    q256 = torch.zeros(2, 4, 136, device="cuda", dtype=BF16)
    k256, v256 = (torch.zeros(3, 2, 16, 136, device="cuda", dtype=BF16) for _ in range(2))
    small = torch.zeros(256, dtype=torch.uint8, device="cuda")
    off = torch.zeros(2 * 4 * 64 + 1, dtype=BF16, device="cuda")[1:].view(2, 4, 64)      # (copied to the workspace first)
    for f, code in ((lambda: ubp.ubp_attention(q, k, v, t, n, scale=0.0), -1), (lambda: ubp.ubp_attention(q, k, v, t, n, scale=float("nan")), -1),
                    (lambda: ubp.ubp_attention(q, k, v, t, n, max_new=0), -1), (lambda: ubp.ubp_attention(q, k7, v7, t, n), -6),
                    (lambda: ubp.ubp_attention(q9, k9, v9, t, n), -6), (lambda: ubp.ubp_attention(q256, k256, v256, t, n), -6),
                    (lambda: ubp.ubp_attention(q, ko, vo, t, n), -1), (lambda: ubp.ubp_prefix_attention(q, k, v, t, n, -1), -1),
                    (lambda: ubp.ubp_prefix_attention(q, k, v, t, n, 16 * t.shape[1] + 1), -1), (lambda: ubp.ubp_attention(off, k, v, t, n, workspace=small), -3)):
        with pytest.raises(ubp.UbpError) as e:
            f()
        assert e.value.code == code
