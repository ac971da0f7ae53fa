"""Norm with the residual's addition and 8-bit rows, and rows to 8 bits, against the formulas in 64 bits."""
import pytest
import torch

from linear_ref import F8, SCALE_MIN, TINY, UNIT, e4m3_half_step

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
EPS = 1e-5


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


def rows_in(T, C, dtype, pad, seed, lead=0):
    """[T][C] rows inside a wider buffer that starts `lead` elements past an allocation's start."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((T * (C + pad) + lead,), float("nan"), device="cuda", dtype=dtype)
    v = buf[lead:].view(T, C + pad)[:, :C]
    v.copy_(torch.randn(T, C, device="cuda", generator=g) * torch.exp(torch.randn(T, 1, device="cuda", generator=g)))
    return v


def norm64(h, gamma):
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    return h * gamma * r


def rel_tol(C):
    """Sum of C squares, each thread adding at most C / 32 of them one after the other: relative error (C / 32 + 16) 2^-24,
    half of it in the inverse root; eight more roundings (root, products, division)."""
    return (C / 64.0 + 16.0) * 2.0 ** -24


def check_q(q, s, y, tol):
    """8-bit rows against their exact values y (64 bits): the scale to `tol`, each code to half a step around the exact
    quotient (the quotient itself may be off by 2 tol)."""
    s64 = (y.abs().amax(1) / 448.0).clamp_min(SCALE_MIN)
    assert ((s.double() - s64).abs() <= tol * s64).all()
    v = y / s64[:, None]
    assert ((q.double() - v).abs() <= e4m3_half_step(v) * (1 + 1e-9) + 3 * tol * v.abs() + 2.0 ** -140).all()
    assert (q.double().abs().amax(1)[y.abs().amax(1) > 448 * SCALE_MIN] == 448).all()      # the largest value gets the largest code


SHAPES = [(1, 1), (3, 7), (1, 4096), (5, 64), (7, 100), (33, 513), (200, 1024), (9, 2051), (4, 8192), (3, 16384), (2, 16392), (2, 40000), (2, 9001),
          (1300, 1500), (3, 2560), (700, 2561), (2, 4097), (310, 5120), (310, 5121), (160, 8191), (150, 8193), (2, 10240), (2, 10241),
          (1300, 800), (5300, 1000), (310, 4000)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,C", SHAPES)
@pytest.mark.parametrize("pad,lead", [(0, 0), (8, 8), (3, 1)])
def test_norm(ubp, dtype, T, C, pad, lead):
    x, r = rows_in(T, C, dtype, pad, 1, lead), rows_in(T, C, dtype, pad, 2, lead)
    gamma = (1 + 0.2 * torch.randn(C, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))).to(dtype)
    want_h = (x.float() + r.float())
    h64, h32 = x.double() + r.double(), want_h.double()
    y64 = norm64(h64, gamma.double())
    tol = rel_tol(C) + 2.0 ** -23                       # (+ the sum x + r itself, rounded to fp32)
    slack = 2.0 ** -23 * (x.double().abs() + r.double().abs()) * gamma.double().abs() * torch.rsqrt((h64 * h64).mean(1, keepdim=True) + EPS)
    y, s, h = ubp.ubp_rmsnorm(x, gamma, EPS, residual=r)
    assert s is None and y.dtype == dtype and torch.equal(h, want_h.to(dtype))
    assert ((y.double() - y64).abs() <= (tol + UNIT[dtype]) * y64.abs() + slack + TINY[dtype]).all()
    q, s, h = ubp.ubp_rmsnorm(x, gamma, EPS, residual=r, out_dtype=F8)
    assert torch.equal(h, want_h.to(dtype))
    check_q(q, s, norm64(h32, gamma.double()), rel_tol(C) + 2.0 ** -22)
    # without a residual; fp32 gamma
    y, _, h = ubp.ubp_rmsnorm(x, gamma.float(), EPS)
    y64 = norm64(x.double(), gamma.double())
    assert h is None and ((y.double() - y64).abs() <= (tol + UNIT[dtype]) * y64.abs() + TINY[dtype]).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,C", SHAPES)
@pytest.mark.parametrize("pad,lead", [(0, 0), (8, 8), (3, 1)])
def test_quant_rows(ubp, dtype, T, C, pad, lead):
    x = rows_in(T, C, dtype, pad, 5, lead)
    q, s = ubp.ubp_quant_rows(x)
    check_q(q, s, x.double(), 2.0 ** -22)


def test_output_strides_and_padding(ubp):
    x = rows_in(6, 72, torch.bfloat16, 0, 7)
    buf = torch.full((6, 80), 1.0, device="cuda").to(F8)
    q = buf[:, :72]
    _, s = ubp.ubp_quant_rows(x, out=q)
    want, want_s = ubp.ubp_quant_rows(x)
    assert torch.equal(q.float(), want.float()) and torch.equal(s, want_s)
    assert (buf[:, 72:].float() == 1.0).all()
    ybuf = torch.full((6, 75), 5.0, device="cuda", dtype=torch.bfloat16)
    gamma = torch.ones(72, device="cuda", dtype=torch.bfloat16)
    ubp.ubp_rmsnorm(x, gamma, EPS, out=ybuf[:, :72])
    assert torch.equal(ybuf[:, :72], ubp.ubp_rmsnorm(x, gamma, EPS)[0]) and (ybuf[:, 72:] == 5.0).all()


@pytest.mark.parametrize("C", [64, 1001, 8192, 50000])
def test_sum_written_over_an_input(ubp, C):
    for which in ("x", "residual"):
        x, r = rows_in(9, C, torch.bfloat16, 0, 11), rows_in(9, C, torch.bfloat16, 0, 12)
        gamma = torch.ones(C, device="cuda", dtype=torch.bfloat16)
        want = ubp.ubp_rmsnorm(x, gamma, EPS, residual=r, out_dtype=F8)
        got = ubp.ubp_rmsnorm(x, gamma, EPS, residual=r, out_dtype=F8, residual_out=x if which == "x" else r)
        assert got[2] is (x if which == "x" else r)
        for a, b in zip(want, got):
            assert torch.equal(a.float(), b.float())


def test_zero_rows_and_special_values(ubp):
    for C in (64, 65):
        x = torch.randn(5, C, device="cuda").to(torch.bfloat16)
        x[1] = 0
        x[2, 3] = float("nan")
        x[3, 5] = float("inf")
        q, s = ubp.ubp_quant_rows(x)
        assert s[1].item() == SCALE_MIN and (q[1].float() == 0).all()
        assert s[2].isnan() and q[2].float().isnan().all()
        assert s[3].isinf() and torch.isfinite(q[0].float()).all() and torch.isfinite(q[4].float()).all()
        gamma = torch.ones(C, device="cuda", dtype=torch.bfloat16)
        q, s, _ = ubp.ubp_rmsnorm(x, gamma, 0.0, out_dtype=F8)
        assert s[2].isnan() and s[3].isnan() and torch.isfinite(s[[0, 4]]).all() and torch.isfinite(q[[0, 4]].float()).all()
        q, s, _ = ubp.ubp_rmsnorm(x, gamma, EPS, out_dtype=F8)
        assert s[1].item() == SCALE_MIN and (q[1].float() == 0).all()
    tiny = torch.full((2, 64), 2.0 ** -133, device="cuda", dtype=torch.bfloat16)      # subnormal: below the smallest scale's grid
    q, s = ubp.ubp_quant_rows(tiny)
    assert (s == SCALE_MIN).all() and (q.float() == 2.0 ** -7).all()


def test_no_rows(ubp):
    x = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    q, s = ubp.ubp_quant_rows(x)
    assert q.shape == (0, 64) and s.shape == (0,)
    y, s, h = ubp.ubp_rmsnorm(x, torch.ones(64, device="cuda", dtype=torch.bfloat16), residual=x, out_dtype=F8)
    assert y.shape == (0, 64) and s.shape == (0,) and h.shape == (0, 64)


def test_offsets_beyond_32_bits(ubp):
    ld = (1 << 30) + 8
    buf = torch.empty(3 * ld, dtype=torch.bfloat16, device="cuda")
    x = buf.view(3, ld)[:, :1000]
    x.copy_(torch.randn(3, 1000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)))
    q, s = ubp.ubp_quant_rows(x)
    want, ws = ubp.ubp_quant_rows(x.contiguous())
    assert torch.equal(q.float(), want.float()) and torch.equal(s, ws)


def test_other_stream(ubp):
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        x = torch.randn(4096, 4096, device="cuda").to(torch.bfloat16)
        for _ in range(10):
            x = x * 1.0
        q, s = ubp.ubp_quant_rows(x)
    st.synchronize()
    want, ws = ubp.ubp_quant_rows(x)
    assert torch.equal(q.float(), want.float()) and torch.equal(s, ws)


def test_refusals(ubp):
    x = torch.randn(4, 64, device="cuda", dtype=torch.bfloat16)
    g = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    bad = [lambda: ubp.ubp_rmsnorm(x.double(), g), lambda: ubp.ubp_rmsnorm(x, g[:63]), lambda: ubp.ubp_rmsnorm(x, g.half()),
           lambda: ubp.ubp_rmsnorm(x, g, residual=x[:3]), lambda: ubp.ubp_rmsnorm(x, g, residual=x.float()),
           lambda: ubp.ubp_rmsnorm(x.t(), g), lambda: ubp.ubp_rmsnorm(x, g, out_dtype=torch.float32),
           lambda: ubp.ubp_rmsnorm(x.cpu(), g), lambda: ubp.ubp_rmsnorm(x, g, out_dtype=F8, scales=torch.empty(3, device="cuda")),
           lambda: ubp.ubp_rmsnorm(x, g, residual=x[:1].expand(4, 64)), lambda: ubp.ubp_quant_rows(x[0]),
           lambda: ubp.ubp_quant_rows(x.to(F8)), lambda: ubp.ubp_quant_rows(x, out=torch.empty(4, 64, device="cuda"))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(ubp.UbpError) as e:
        ubp.ubp_rmsnorm(x, g, eps=-1.0)
    assert e.value.code == -1
