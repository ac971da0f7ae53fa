"""8-bit codes of the row operators against the fp32 quotient, and single rows cut from wider buffers."""
import pytest
import torch

from linear_ref import F8

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
IDS = ["bf16", "f16", "f32"]


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


def scales(v):
    """max |v| / 448 of each row, divided (torch multiplies by the reciprocal where the divisor is a number, not a tensor)."""
    m = v.float().abs().amax(1)
    return (m / torch.full_like(m, 448.0)).clamp_min(2.0 ** -126)


def codes(v, s):
    """e4m3(v / s) with the quotient rounded to fp32 first (IEEE division)."""
    return (v.float() / s[:, None]).to(F8).view(torch.uint8)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("T,C,pad", [(4001, 4096, 0), (1531, 2051, 3), (700, 16384, 8), (300, 20001, 1), (9000, 250, 0), (64, 40000, 0), (400, 5121, 1), (300, 8191, 1),
                                     (300, 9001, 1), (300, 10241, 1), (200, 16383, 2)])
def test_codes_are_the_rounded_quotients(ubp, dtype, T, C, pad):
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.empty(T, C + pad, device="cuda", dtype=dtype)[:, :C]
    x.copy_(torch.randn(T, C, device="cuda", generator=g) * torch.exp(torch.randn(T, C, device="cuda", generator=g)))
    q, s = ubp.ubp_quant_rows(x)
    assert torch.equal(s, scales(x))
    assert torch.equal(q.view(torch.uint8), codes(x, s))


def test_a_code_beside_a_midpoint(ubp):
    """6.3121e-05 / (0.689453125 / 448) lies just below the midpoint of the codes 0.0390625 and 0.04296875."""
    for C in (64, 65):
        x = torch.zeros(2, C, device="cuda", dtype=torch.float16)
        x[:, 0], x[:, 1] = 0.689453125, 6.3121e-05
        q, s = ubp.ubp_quant_rows(x)
        assert torch.equal(q.view(torch.uint8), codes(x, s)) and q[0, 1].item() == 0.0390625


@pytest.mark.parametrize("C,pad", [(512, 0), (1001, 1), (20000, 0)])
def test_codes_over_the_whole_range_of_scales(ubp, C, pad):
    """Rows from the smallest numbers to the largest: scales from 2^-126 to 2^119, subnormal quotients and values among them."""
    g = torch.Generator(device="cuda").manual_seed(C)
    e = torch.arange(-149, 126, device="cuda")
    x = torch.randn(e.numel(), C, device="cuda", generator=g) * torch.exp(2 * torch.randn(e.numel(), C, device="cuda", generator=g))
    x = torch.ldexp(x.double(), e[:, None]).clamp(-3e38, 3e38)
    for dtype in (torch.bfloat16, torch.float32):
        v = torch.empty(e.numel(), C + pad, device="cuda", dtype=dtype)[:, :C]
        v.copy_(x.to(dtype))
        q, s = ubp.ubp_quant_rows(v)
        assert torch.equal(s, scales(v))
        assert torch.equal(q.view(torch.uint8), codes(v, s))


@pytest.mark.parametrize("T,C,pad", [(300, 4096, 0), (200, 2051, 3), (9, 20000, 0), (500, 96, 0), (7, 8192, 0)])
def test_codes_of_the_norm_are_the_rounded_quotients(ubp, T, C, pad):
    """fp32 rows: the norm in fp32 is what the 8-bit form divides by its scale."""
    g = torch.Generator(device="cuda").manual_seed(C)
    x = torch.empty(T, C + pad, device="cuda")[:, :C]
    x.copy_(torch.randn(T, C, device="cuda", generator=g) * torch.exp(torch.randn(T, C, device="cuda", generator=g)))
    gamma = 1 + 0.2 * torch.randn(C, device="cuda", generator=g)
    for scale in (1.0, 2.0 ** -100):
        y, _, _ = ubp.ubp_rmsnorm(x, gamma * scale, 1e-5, out=torch.empty(T, C + pad, device="cuda")[:, :C])
        q, s, _ = ubp.ubp_rmsnorm(x, gamma * scale, 1e-5, out_dtype=F8)
        assert torch.equal(s, scales(y))
        assert torch.equal(q.view(torch.uint8), codes(y, s))


def test_infinite_rows(ubp):
    """A row with an infinity has an infinite scale: its finite values are 0, the infinity is NaN, as the quotients are."""
    for C in (64, 65, 20000, 20001):
        x = torch.randn(3, C, device="cuda")
        x[1, 5] = float("inf")
        q, s = ubp.ubp_quant_rows(x)
        assert s[1].isinf() and torch.equal(q.float().nan_to_num(7.0), codes(x, s).view(F8).float().nan_to_num(7.0))


@pytest.mark.parametrize("C", [96, 1000, 4096, 8192])
def test_one_row_of_a_wider_buffer(ubp, C):
    """The pitch of a single row says nothing about its alignment: the same kernel as for a contiguous row, the same bits."""
    for seed in range(8):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def row(v):
            b = torch.empty(2, C + 3, device="cuda")
            b[0, :C] = v
            return b[:1, :C]

        x, r = (torch.randn(1, C, device="cuda", generator=g) for _ in range(2))
        gamma = torch.ones(C, device="cuda")
        want, _, h = ubp.ubp_rmsnorm(x, gamma, 1e-5, residual=r)
        got, _, h1 = ubp.ubp_rmsnorm(row(x), gamma, 1e-5, residual=row(r), out=row(0.0), residual_out=row(0.0))
        assert torch.equal(got, want) and torch.equal(h1, h)


def test_rows_without_a_norm(ubp):
    """eps = 0: a row of zeros is 0 / 0, one whose squares vanish in fp32 is not finite; a positive eps gives zeros their zeros."""
    for C in (64, 65):
        x = torch.randn(3, C, device="cuda")
        x[1], x[2] = 0, 1e-30
        gamma = torch.ones(C, device="cuda")
        for out in (torch.float32, F8):
            y, s, _ = ubp.ubp_rmsnorm(x, gamma, 0.0, out_dtype=out)
            y = y.float()
            assert torch.isfinite(y[0]).all() and y[1].isnan().all() and not torch.isfinite(y[2]).any()
            y, s, _ = ubp.ubp_rmsnorm(x, gamma, 1e-6, out_dtype=out)
            assert (y.float()[1] == 0).all() and torch.isfinite(y.float()).all()


def test_no_gradient_is_recorded(ubp):
    x = torch.randn(3, 64, device="cuda", requires_grad=True)
    gamma = torch.ones(64, device="cuda", requires_grad=True)
    assert not any(t.requires_grad for t in ubp.ubp_rmsnorm(x, gamma, 1e-5, residual=x, out_dtype=F8) + ubp.ubp_quant_rows(x))
