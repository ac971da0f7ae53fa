"""Values of the token-major product where forms and types could differ: fp32 outputs, infinities and NaN in x, outputs over inputs."""
import pytest
import torch

from linear_ref import F8, make_weight

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
IDS = {BF16: "bf16", F16: "f16", F8: "e4m3"}


@pytest.fixture(scope="module")
def ubp():
    import paper_2407_19644_b200 as m
    m.load()
    return m


def act64(v, act):
    """The activation in 64 bits (erfc instead of 1 + erf, which loses the digits of the negative tail) and the relative error
    that fp32 may have: CUDA states 5 units in the last place (of 2^-23) for the normal distribution function and 2 for expf;
    the products, the sum and the division add half a unit each. The argument of gelu_tanh, a product of rounded constants and
    a sum of rounded powers, is off by at most 6 roundings, which the exponential turns into that times the argument."""
    u = 2.0 ** -23
    if act == "gelu":
        return 0.5 * v * torch.erfc(-v / 2.0 ** 0.5), torch.full_like(v, 6 * u)
    if act == "silu":
        return v * torch.sigmoid(v), torch.full_like(v, 4 * u)
    a = 2.0 * (2.0 / torch.pi) ** 0.5 * (v + 0.044715 * v ** 3)
    return v * torch.sigmoid(a), 4 * u + 3 * u * a.abs() * torch.sigmoid(-a)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("T", [1, 40, 40000])
def test_fp32_outputs_have_fp32_activations(ubp, act, T):
    v = torch.cat([torch.linspace(-12, 12, 1501), torch.linspace(-1, 1, 501), torch.tensor([-90.0, -40.0, -20.0, 20.0, 90.0, 1e4, -1e4, 0.0, 3e38, -3e38])]).cuda()
    if T > 1000:
        v = v[::40].contiguous()                       # (few enough rows for the pair kernel to be chosen)
    F = v.numel()
    want, rel = act64(v.double(), act)
    for gated in (False, True):
        M = 2 * F if gated else F
        W, mask = make_weight(M, 64, 1, 50, 5)
        b = torch.cat([v, torch.ones_like(v)]) if gated else v
        plan = ubp.LinearPlan(ubp.ubp_pack(W, mask, 1), BF16, gated=gated)
        y = ubp.ubp_linear(plan, torch.zeros(T, 64, device="cuda", dtype=BF16), bias=b, activation=act, out_dtype=torch.float32)
        assert plan.choice(T)[0] == {1: 0, 40: 1, 40000: 2}[T]
        err = (y.double() - want).abs()
        bound = rel * want.abs() + 2.0 ** -118
        assert (err <= bound).all(), float((err / bound).max())
