"""Head norms with the position rotation and the append to a paged cache, against the formulas in 64 bits."""
import pytest
import torch

from attention_ref import BF16, F16, Batch, rand
from linear_ref import TINY, UNIT

pytestmark = pytest.mark.gpu

EPS = 1e-6


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


def rows_in(b, width, pad, lead, extra=0):
    buf = torch.full(((b.T + extra) * (width + pad) + lead,), float("nan"), device="cuda", dtype=b.dtype)
    v = buf[lead:].view(b.T + extra, width + pad)[:, :width]
    v.copy_(rand(b.g, b.T + extra, width) * torch.exp(rand(b.g, b.T + extra, 1)))
    return v


def turned(x, rotation, positions, interleaved):
    """x [n][H][D] and the sizes of what is added for each value."""
    r = rotation.shape[1]
    c, s = rotation[positions].double()[:, None].chunk(2, dim=2)
    y, size = x.clone(), x.abs()
    i, j = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y[:, :, i], y[:, :, j] = x[:, :, i] * c - x[:, :, j] * s, x[:, :, j] * c + x[:, :, i] * s
    size[:, :, i], size[:, :, j] = (x[:, :, i] * c).abs() + (x[:, :, j] * s).abs(), (x[:, :, j] * c).abs() + (x[:, :, i] * s).abs()
    return y, size


def check(ubp, b, qkv, rotation, interleaved, qg, kg, q_out=None):
    Hq, Hkv, D, u = b.Hq, b.Hkv, b.D, UNIT[b.dtype]
    x = qkv.double().unflatten(1, (Hq + 2 * Hkv, D))
    before = b.k.clone(), b.v.clone()
    raw = qkv.clone()
    q = ubp.ubp_rotate_append(qkv, Hq, *b.args(), starts=b.starts, rotation=rotation, interleaved=interleaved, q_gamma=qg, k_gamma=kg, eps=EPS, out=q_out)
    # D squares summed in any order, half of that error in the root; root, quotient, three products, one sum; at most 2^-23 each
    tol = (D / 2 + 12) * 2.0 ** -23
    touched = torch.zeros(b.k.shape[0], b.page, dtype=torch.bool, device="cuda")
    for s, (a, n) in enumerate(zip(b.new, b.lengths)):
        t = b.first[s]
        p = torch.arange(n - a, n, device="cuda")
        y = x[t:t + a, :Hq + Hkv]
        for part, g in ((slice(0, Hq), qg), (slice(Hq, Hq + Hkv), kg)):
            if g is not None:
                z = y[:, part]
                y = y.clone()
                y[:, part] = z * torch.rsqrt((z * z).mean(2, keepdim=True) + EPS) * g.double()
        y, size = (y, y.abs()) if rotation is None else turned(y, rotation, p, interleaved)
        bound = tol * size + u * y.abs() + TINY[b.dtype]
        assert ((q[t:t + a].double() - y[:, :Hq]).abs() <= bound[:, :Hq]).all()
        page, slot = b.table[s].long()[p // b.page], p % b.page
        assert ((b.k[page, :, slot].double() - y[:, Hq:]).abs() <= bound[:, Hq:]).all()
        assert torch.equal(b.v[page, :, slot], raw.unflatten(1, (Hq + 2 * Hkv, D))[t:t + a, Hq + Hkv:])
        touched[page, slot] = True
    for now, old in ((b.k, before[0]), (b.v, before[1])):       # nothing else is written
        now, old = now.transpose(1, 2)[~touched], old.transpose(1, 2)[~touched]
        assert torch.equal(now.view(torch.int16), old.view(torch.int16))
    return q


LAYOUTS = [(4, 2, 64, 64, False), (32, 8, 128, 128, False), (12, 4, 80, 32, True), (3, 3, 96, 96, True), (8, 1, 128, 64, False), (5, 1, 72, 20, False),
           (2, 1, 8, 8, False), (6, 2, 80, 40, False), (7, 7, 128, 128, True), (1, 1, 16, 16, False), (4, 4, 112, 2, True)]


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("Hq,Hkv,D,r,interleaved", LAYOUTS)
@pytest.mark.parametrize("norm", ["both", "none", "keys"])
@pytest.mark.parametrize("pad,lead", [(0, 0), (8, 8), (3, 1)])
def test_layouts(ubp, dtype, Hq, Hkv, D, r, interleaved, norm, pad, lead):
    for new, lengths, single in (([1], [70], True), ([1, 1, 1], [5, 1, 200], True), ([0, 7, 40, 0, 1], [3, 7, 95, 0, 64], False)):
        b = Batch(new, lengths, Hq, Hkv, D, dtype, [8, 16, 64][(Hq + pad) % 3], seed=D + pad, behind=0 if single else 2, single=single)
        qkv = rows_in(b, (Hq + 2 * Hkv) * D, pad, lead)
        rotation = ubp.rotation_table(max(lengths), r)
        qg, kg = ((1 + 0.2 * rand(b.g, D)).to(dtype) for _ in range(2))
        check(ubp, b, qkv, rotation, interleaved, qg if norm == "both" else None, kg if norm != "none" else None)
        check(ubp, b, qkv, None, interleaved, None, kg if norm != "none" else None)


@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_many_tokens_and_in_place(ubp, layout):
    b = Batch([1500, 0, 900], [1500, 7, 1000], 8, 2, 64, BF16, 16, layout=layout)
    qkv = rows_in(b, 12 * 64, 0, 0)
    g = (1 + 0.2 * rand(b.g, 64)).to(BF16)
    rotation = ubp.rotation_table(2000, 64)
    q = check(ubp, b, qkv.clone(), rotation, False, g, g)
    own = qkv.clone()
    check(ubp, b, own, rotation, False, g, g, q_out=own[:, :8 * 64].unflatten(1, (8, 64)))
    assert torch.equal(own[:, :8 * 64], q.flatten(1)) and torch.equal(own[:, 8 * 64:], qkv[:, 8 * 64:])


def test_many_sequences(ubp):
    n = 1500
    new = [b * 7 % 3 for b in range(n)]
    b = Batch(new, [a + b % 11 for b, a in enumerate(new)], 2, 1, 32, F16, 8, behind=5)
    check(ubp, b, rows_in(b, 4 * 32, 0, 0), ubp.rotation_table(20, 32), False, None, None)


def test_rotation_table_far_positions(ubp):
    """Angles of far positions, against a table made value by value in Python's doubles."""
    import math
    t = ubp.rotation_table(200001, 8, base=500.0, scale=0.5).cpu()
    for p in (0, 1, 77777, 200000):
        for i in range(4):
            x = p * 0.5 * 500.0 ** (-2 * i / 8)
            assert abs(t[p, i].item() - math.cos(x)) <= 2.0 ** -24 + 1e-10 and abs(t[p, 4 + i].item() - math.sin(x)) <= 2.0 ** -24 + 1e-10
    with pytest.raises(ValueError):
        ubp.rotation_table(10, 7)


def test_places_that_do_not_exist(ubp):
    """Positions before the sequence or without a rotation: queries 0, nothing appended. Pages outside the cache: not appended."""
    for pad in (0, 3):
        b = Batch([3, 2, 1], [40, 2, 60], 2, 1, 64, BF16, 16)
        qkv = rows_in(b, 4 * 64, pad, 0)
        b.len_t[1] = 1                                                      # one of its two tokens lies before position 0
        b.table[2, 3] = b.k.shape[0]
        old = b.k.clone()
        q = ubp.ubp_rotate_append(qkv, 2, *b.args(), starts=b.starts, rotation=ubp.rotation_table(39, 64))
        assert (q[2] == 0).all() and (q[3] == 0).all() and (q[5] == 0).all() and (q[[0, 1, 4]] != 0).any(2).all()
        changed = (b.k.view(torch.int16) != old.view(torch.int16)).any(3).sum()
        assert changed == 3                                                 # positions 37, 38 and 0
        old = b.k.clone()
        q = ubp.ubp_rotate_append(qkv, 2, *b.args(), starts=b.starts)       # no rotation: only the page is missing now
        assert (q[5] != 0).any() and (q[3] == 0).all()
        page = b.table[0, 39 // 16].long()
        assert torch.equal(b.k[page, 0, 39 % 16], qkv[2, 128:192])


def test_captured_call_follows_the_lengths(ubp):
    b = Batch([1, 1], [30, 50], 2, 1, 64, BF16, 16, single=True)
    qkv = rows_in(b, 4 * 64, 0, 0)
    rotation = ubp.rotation_table(64, 64)
    g = torch.cuda.CUDAGraph()
    ubp.ubp_rotate_append(qkv, 2, *b.args(), rotation=rotation)
    with torch.cuda.graph(g):
        q = ubp.ubp_rotate_append(qkv, 2, *b.args(), rotation=rotation)
    for lengths in ([30, 50], [7, 49], [32, 33]):
        b.len_t.copy_(torch.tensor(lengths, dtype=torch.int32))
        g.replay()
        got = q.clone()
        assert torch.equal(got, ubp.ubp_rotate_append(qkv, 2, *b.args(), rotation=rotation))
        for s, n in enumerate(lengths):
            assert torch.equal(b.v[b.table[s, (n - 1) // 16].long(), 0, (n - 1) % 16], qkv[s, 192:])


def test_refusals(ubp):
    b = Batch([1, 1], [40, 40], 4, 2, 64, BF16, 16)
    qkv = rows_in(b, 8 * 64, 0, 0)
    k, v, t, n = b.args()
    rot, g = ubp.rotation_table(64, 64), torch.ones(64, dtype=BF16, device="cuda")
    bad = [lambda: ubp.ubp_rotate_append(qkv[:, :-1], 4, k, v, t, n), lambda: ubp.ubp_rotate_append(qkv, 3, k, v, t, n), lambda: ubp.ubp_rotate_append(qkv.half(), 4, k, v, t, n),
           lambda: ubp.ubp_rotate_append(qkv, 4, k, v[:1], t, n), lambda: ubp.ubp_rotate_append(qkv, 4, k, v, t, n, rotation=rot.double()),
           lambda: ubp.ubp_rotate_append(qkv, 4, k, v, t, n, rotation=rot[:, :63]), lambda: ubp.ubp_rotate_append(qkv, 4, k, v, t, n, rotation=ubp.rotation_table(9, 66)),
           lambda: ubp.ubp_rotate_append(qkv, 4, k, v, t, n, q_gamma=g[:63]), lambda: ubp.ubp_rotate_append(qkv, 4, k, v, t, n, k_gamma=g.float()),
           lambda: ubp.ubp_rotate_append(qkv[:1], 4, k, v, t, n), lambda: ubp.ubp_rotate_append(qkv, 4, k, v, t, n, out=torch.empty(2, 4, 63, dtype=BF16, device="cuda")),
           lambda: ubp.ubp_rotate_append(qkv, 4, k, v, t, n, starts=n), lambda: ubp.ubp_rotate_append(qkv, 4, k, v, t.cpu(), n)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(ubp.UbpError) as e:
        ubp.ubp_rotate_append(qkv, 4, k, v, t, n, eps=-1.0)
    assert e.value.code == -1
