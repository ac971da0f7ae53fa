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


def without_rows(W, mask, Nb, n):
    """The layer without the blocks that start in its first n rows."""
    mask = mask.copy()
    for j in range(mask.shape[1]):
        i = n
        while i < mask.shape[0] and mask[i, j]:
            i += 1
        mask[:n + (i - n) % Nb, j] = 0
    return W * mask, mask


@pytest.mark.parametrize("dtype", [BF16, F16, F8], ids=IDS.get)
@pytest.mark.parametrize("T", [1, 2, 5, 16])
@pytest.mark.parametrize("M,C,Nb,gated", [(512, 512, 8, False), (640, 300, 4, True), (300, 1003, 2, False), (256, 256, 3, False)])
def test_kept_blocks_alone_see_infinities(ubp, dtype, T, M, C, Nb, gated):
    """The kept-block kernel multiplies kept weights only: an infinity or NaN in a channel reaches the outputs that keep this
    channel, as the product with their weight, and no other; rows without blocks stay what they are."""
    W, mask = make_weight(M, C, Nb, 90, 9)
    W, mask = without_rows(W, mask, Nb, 48)            # whole rows empty, beside rows that are not
    plan = ubp.LinearPlan(ubp.ubp_pack(W, mask, Nb), dtype, gated=gated)
    assert plan.choice(T)[0] == 0
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, C, device="cuda", generator=g).to(dtype)
    xs = torch.ones(T, device="cuda") if dtype == F8 else None
    kept = torch.from_numpy(mask != 0).cuda()
    w = torch.from_numpy(W).cuda().double()
    t = T - 1
    specials = [(0, "nan"), (C - 1, "nan")] + ([] if dtype == F8 else [(0, "inf"), (C - 1, "inf"), (C // 2, "-inf")])
    for j, v in specials:
        zeroed, bad = x.clone(), x.clone()
        zeroed[t, j] = 0.0
        bad[t, j] = float(v)
        z = ubp.ubp_linear(plan, zeroed, x_scales=xs, out_dtype=torch.float32).double()
        y = ubp.ubp_linear(plan, bad, x_scales=xs, out_dtype=torch.float32).double()
        want = z.clone()
        add = torch.where(kept[:, j], w[:, j] * float(v), torch.zeros_like(w[:, j]))
        if gated:
            touched = kept[:M // 2, j] | kept[M // 2:, j]
            assert torch.equal(y[t][~touched], z[t][~touched]) and not torch.isfinite(y[t][touched]).any()
        else:
            want[t] += add
            assert torch.equal(y[t].nan_to_num(7.0, 8.0, 9.0), want[t].nan_to_num(7.0, 8.0, 9.0))
        assert torch.equal(y[:t], z[:t])
    if dtype != F8 and not gated:                      # every channel infinite: each output is its weights' infinities
        bad = torch.full_like(x, float("inf"))
        y = ubp.ubp_linear(plan, bad, out_dtype=torch.float32)
        pos, neg = ((w > 0) & kept).any(1), ((w < 0) & kept).any(1)
        zero = ((w.to(dtype) == 0) & kept).any(1)
        assert (y[:, pos & ~neg & ~zero] == float("inf")).all() and (y[:, neg & ~pos & ~zero] == float("-inf")).all()
        assert y[:, pos & neg].isnan().all() and (y[:, ~kept.any(1)] == 0).all()


def test_outputs_over_inputs(ubp):
    """Every output reads a whole row of x: writing over x is refused. The residual may be the output, with its stride."""
    W, mask = make_weight(128, 128, 4, 50, 1)
    for T in (1, 5, 40):
        plan = ubp.LinearPlan(ubp.ubp_pack(W, mask, 4), BF16)
        x = torch.randn(T, 128, device="cuda").to(BF16)
        with pytest.raises(ValueError):
            ubp.ubp_linear(plan, x, out=x)
    buf = torch.zeros(5, 256, device="cuda", dtype=BF16)
    with pytest.raises(ValueError):
        ubp.ubp_linear(plan, x[:5].clone(), residual=buf[:, :128], out=buf.view(-1)[:640].view(5, 128))
    gamma = torch.ones(128, device="cuda", dtype=BF16)
    rows, tight = buf[:, :128], buf.view(-1)[:640].view(5, 128)
    for bad in (lambda: ubp.ubp_rmsnorm(rows, gamma, residual=x[:5], residual_out=tight), lambda: ubp.ubp_rmsnorm(x[:5], gamma, residual=rows, residual_out=tight),
                lambda: ubp.ubp_rmsnorm(x[:5], gamma, residual=rows, residual_out=tight, out=tight)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("T", [1, 40, 40000])
@pytest.mark.parametrize("out", [BF16, F16], ids=IDS.get)
def test_16_bit_outputs_of_activations(ubp, act, T, out):
    """One rounding of the output on top of the activation's own error: 105 units of 2^-23 of __expf at its largest argument (CUDA:
    2 + 1.173 |x|), the exponent's rounding 88 x 2^-24 at most, the fit and the rest a few units: below 2^-15 in all. Below
    2^-118 the forms may give 0."""
    v = torch.cat([torch.linspace(-12, 12, 1501), torch.linspace(-1, 1, 501), torch.tensor([-90.0, -40.0, -20.0, 20.0, 90.0, 1e4, -1e4, 0.0])]).cuda()
    if T > 1000:
        v = v[::40].contiguous()
    W, mask = make_weight(v.numel(), 64, 1, 50, 5)
    plan = ubp.LinearPlan(ubp.ubp_pack(W, mask, 1), out)
    y = ubp.ubp_linear(plan, torch.zeros(T, 64, device="cuda", dtype=out), bias=v, activation=act).double()
    assert plan.choice(T)[0] == {1: 0, 40: 1, 40000: 2}[T]
    want = act64(v.double(), act)[0]
    unit, tiny = (2.0 ** -8, 2.0 ** -118) if out == BF16 else (2.0 ** -11, 2.0 ** -25)
    err = (y - want).abs()
    bound = (unit + 2.0 ** -15) * want.abs() + tiny
    assert (err <= bound).all(), float((err / bound).max())
